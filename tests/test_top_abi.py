"""grpo_top.h as seen from the host (CPU only): symbols, refusals, workspace sizes; and the binding's own checks.

Every call here fails host-side validation; device pointers are dummies.
"""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2606_05597_amd as grpo
from paper_2606_05597_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = ctypes.c_void_p(0x100000)
ODD = ctypes.c_void_p(0x100001)
FOUR = ctypes.c_void_p(0x100004)
NAMES = ["grpo_token_logp_top_workspace_bytes", "grpo_token_logp_top", "grpo_token_logp_top_bwd"]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.SO):
        from paper_2606_05597_amd.build import build
        build()
    return _lib.load()


def test_header_and_exports(lib, tmp_path):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "grpo_top.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"^\s*(?:int|size_t)\s+(\w+)\s*\(", src, flags=re.M))) == sorted(NAMES)
    out = subprocess.check_output(["nm", "-D", "--defined-only", _lib.SO], text=True)
    assert set(NAMES) <= {line.split()[-1] for line in out.splitlines() if " T " in line}
    c = tmp_path / "t.c"
    c.write_text('#include "grpo_top.h"\n_Static_assert(sizeof(grpo_top_row) == 24, "row");\nint main(void) { return 0; }\n')
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           "-I" + os.path.join(ROOT, "include"), "-c", str(c), "-o", str(tmp_path / "t.o")])


def top(lib, T=8, V=64, ld=64, dt=_lib.GRPO_BF16, n=4, logits=D, temp=None, all_=1.0, act=D, logp=D, ent=D, ids=D, tlp=D,
        rows=D, flags=None, ws=D, ws_bytes=1 << 40):
    return lib.grpo_token_logp_top(logits, dt, T, V, ld, temp, all_, act, n, logp, ent, ids, tlp, rows, flags, ws, ws_bytes,
                                   None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), _lib.GRPO_ERR_ARG), (dict(act=None), _lib.GRPO_ERR_ARG), (dict(all_=0.0), _lib.GRPO_ERR_ARG),
    (dict(all_=-1.0), _lib.GRPO_ERR_ARG), (dict(all_=float("nan")), _lib.GRPO_ERR_ARG), (dict(all_=2e6), _lib.GRPO_ERR_ARG),
    (dict(T=-1), _lib.GRPO_ERR_SHAPE), (dict(T=1 << 31), _lib.GRPO_ERR_SHAPE), (dict(V=0), _lib.GRPO_ERR_SHAPE),
    (dict(ld=63), _lib.GRPO_ERR_SHAPE), (dict(V=(1 << 22) + 1, ld=1 << 23), _lib.GRPO_ERR_SHAPE),
    (dict(n=-1), _lib.GRPO_ERR_SHAPE), (dict(n=65), _lib.GRPO_ERR_SHAPE), (dict(dt=9), _lib.GRPO_ERR_DTYPE),
    (dict(logits=ODD), _lib.GRPO_ERR_ALIGN), (dict(temp=ODD), _lib.GRPO_ERR_ALIGN), (dict(act=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(logp=ODD), _lib.GRPO_ERR_ALIGN), (dict(ent=ODD), _lib.GRPO_ERR_ALIGN), (dict(ids=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(tlp=ODD), _lib.GRPO_ERR_ALIGN), (dict(rows=FOUR), _lib.GRPO_ERR_ALIGN), (dict(flags=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(T=1, V=151936, ld=151936, ws=None), _lib.GRPO_ERR_WORKSPACE),
    (dict(T=1, V=151936, ld=151936, ws_bytes=64), _lib.GRPO_ERR_WORKSPACE),
    (dict(T=1, V=151936, ld=151936, ws=ctypes.c_void_p(0x100008)), _lib.GRPO_ERR_ALIGN)])
def test_refusals(lib, kw, status):
    assert top(lib, **kw) == status


def bwd(lib, T=8, V=64, ld=64, dt=_lib.GRPO_BF16, n=4, logits=D, act=D, ids=D, rows=D, dlogp=D, dent=D, dtop=D,
        out=ctypes.c_void_p(0x200000)):
    return lib.grpo_token_logp_top_bwd(logits, dt, T, V, ld, act, n, ids, rows, dlogp, dent, dtop, out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), _lib.GRPO_ERR_ARG), (dict(act=None), _lib.GRPO_ERR_ARG), (dict(rows=None), _lib.GRPO_ERR_ARG),
    (dict(out=None), _lib.GRPO_ERR_ARG), (dict(ids=None), _lib.GRPO_ERR_ARG), (dict(ld=60), _lib.GRPO_ERR_SHAPE),
    (dict(T=-1), _lib.GRPO_ERR_SHAPE), (dict(n=65), _lib.GRPO_ERR_SHAPE), (dict(dt=5), _lib.GRPO_ERR_DTYPE),
    (dict(logits=ODD), _lib.GRPO_ERR_ALIGN), (dict(act=ODD), _lib.GRPO_ERR_ALIGN), (dict(ids=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(rows=FOUR), _lib.GRPO_ERR_ALIGN), (dict(dlogp=ODD), _lib.GRPO_ERR_ALIGN), (dict(dent=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(dtop=ODD), _lib.GRPO_ERR_ALIGN), (dict(out=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(out=ctypes.c_void_p(0x100002)), _lib.GRPO_ERR_ARG), (dict(out=ctypes.c_void_p(0x100080)), _lib.GRPO_ERR_ARG)])
def test_backward_refusals(lib, kw, status):
    assert bwd(lib, **kw) == status


def test_workspace(lib):
    f = lib.grpo_token_logp_top_workspace_bytes
    assert f(-1, 10, 0) == 0 and f(1, 0, 0) == 0 and f(1, (1 << 22) + 1, 0) == 0 and f(1, 151936, 65) == 0
    for T, V in ((0, 151936), (1, 5), (8, 1024), (8000, 151936)):
        assert f(T, V, 20) == 0  # none is needed
    for T in range(1, 300):
        for V in (16385, 151936, 1 << 22):
            for n in (0, 1, 64):
                b = f(T, V, n)
                assert b % 256 == 0 and b <= T * 16 * (24 + 8 * n) + 512  # at most 16 parts to a row


def test_binding_refusals():
    x, a = torch.zeros(4, 32), torch.zeros(4, dtype=torch.int32)
    f = grpo.grpo_token_logp_top
    with pytest.raises(ValueError, match="GPU"):
        f(x, a, 3)
    for n in (-1, 65):
        with pytest.raises(ValueError, match="n must be"):
            f(x, a, n)
    with pytest.raises(ValueError, match="V must be"):
        f(x, a, 3, V=33)
    with pytest.raises(TypeError, match="actions"):
        f(x, a.long(), 3)
    with pytest.raises(ValueError, match="actions"):
        f(x, a[:3], 3)
    with pytest.raises(TypeError, match="logits"):
        f(x.double(), a, 3)
    with pytest.raises(ValueError, match="unit column stride"):
        f(x.t().contiguous().t(), a, 3)
    with pytest.raises(TypeError, match="temperature"):
        f(x, a, 3, temperature=torch.ones(4, dtype=torch.float64))
    with pytest.raises(ValueError, match="temperature"):
        f(x, a, 3, temperature=torch.ones(3))
    g = grpo.grpo_token_logp_top_bwd
    ids, rows, up = torch.zeros((4, 3), dtype=torch.int32), torch.zeros((4, 24), dtype=torch.uint8), torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        g(x, a, ids, rows, up, up)
    with pytest.raises(ValueError, match="ids"):
        g(x, a, ids[:3], rows)
    with pytest.raises(ValueError, match="rows"):
        g(x, a, ids, rows[:, :20])
    with pytest.raises(ValueError, match="dtop"):
        g(x, a, ids, rows, None, None, torch.zeros(4, 2))
    with pytest.raises(ValueError, match="dlogits"):
        g(x, a, ids, rows, up, dlogits=None)
    with pytest.raises(ValueError, match="dlogits"):
        g(x, a, ids, rows, up, dlogits=torch.zeros(4, 31))
