"""grpo_sampling.h and grpo_clip.h as seen from the host (CPU only): symbols, refusals, the clipping's table.

Every call here fails host-side validation or touches host memory alone; device pointers are dummies.
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


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.SO):
        from paper_2606_05597_amd.build import build
        build()
    return _lib.load()


@pytest.mark.parametrize("header,names", [
    ("grpo_sampling.h", ["grpo_sampling_workspace_bytes", "grpo_sample", "grpo_sampled_logp", "grpo_sampled_logp_bwd"]),
    ("grpo_clip.h", ["grpo_grad_table_bytes", "grpo_grad_table", "grpo_grad_sumsq", "grpo_grad_clip"]),
])
def test_headers_and_exports(lib, header, names):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert sorted(set(re.findall(r"^\s*(?:int|size_t)\s+(\w+)\s*\(", src, flags=re.M))) == sorted(names)
    out = subprocess.check_output(["nm", "-D", "--defined-only", _lib.SO], text=True)
    exported = {line.split()[-1] for line in out.splitlines() if " T " in line}
    assert set(names) <= exported


def test_headers_compile_as_c(tmp_path):
    c = tmp_path / "t.c"
    c.write_text('#include "grpo_sampling.h"\n#include "grpo_clip.h"\n'
                 "_Static_assert(sizeof(grpo_sampling_row) == 32, \"row\");\nint main(void) { return 0; }\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           "-I" + os.path.join(ROOT, "include"), "-c", str(c), "-o", str(tmp_path / "t.o")])


def par(**kw):
    p = _lib.Sampling()
    p.temperature_all, p.top_p_all = 1.0, 1.0
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def sample(lib, which="sample", T=8, V=64, ld=64, dt=_lib.GRPO_BF16, p=None, logits=D, u=D, actions=D, logp=D, n=D, rows=D,
           flags=None, ws=D, ws_bytes=1 << 40, no_par=False):
    pp = None if no_par else ctypes.byref(p or par())
    if which == "sample":
        return lib.grpo_sample(logits, dt, T, V, ld, pp, u, actions, logp, n, flags, ws, ws_bytes, None)
    return lib.grpo_sampled_logp(logits, dt, T, V, ld, pp, actions, logp, n, rows, flags, ws, ws_bytes, None)


BAD_SAMPLE = [
    (dict(logits=None), _lib.GRPO_ERR_ARG), (dict(actions=None), _lib.GRPO_ERR_ARG), (dict(no_par=True), _lib.GRPO_ERR_ARG),
    (dict(T=-1), _lib.GRPO_ERR_SHAPE), (dict(T=1 << 31), _lib.GRPO_ERR_SHAPE), (dict(V=0), _lib.GRPO_ERR_SHAPE),
    (dict(ld=63), _lib.GRPO_ERR_SHAPE), (dict(V=(1 << 22) + 1, ld=1 << 23), _lib.GRPO_ERR_SHAPE),
    (dict(dt=7), _lib.GRPO_ERR_DTYPE), (dict(logits=ODD), _lib.GRPO_ERR_ALIGN), (dict(actions=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(logp=ODD), _lib.GRPO_ERR_ALIGN), (dict(n=ODD), _lib.GRPO_ERR_ALIGN), (dict(flags=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(p=par(temperature_all=-1.0)), _lib.GRPO_ERR_ARG), (dict(p=par(temperature_all=float("nan"))), _lib.GRPO_ERR_ARG),
    (dict(p=par(temperature_all=1e-7)), _lib.GRPO_ERR_ARG), (dict(p=par(temperature_all=2e6)), _lib.GRPO_ERR_ARG),
    (dict(p=par(top_p_all=1.5)), _lib.GRPO_ERR_ARG), (dict(p=par(top_p_all=float("nan"))), _lib.GRPO_ERR_ARG),
    (dict(p=par(min_p_all=-0.5)), _lib.GRPO_ERR_ARG), (dict(p=par(top_k=0x100001)), _lib.GRPO_ERR_ALIGN),
    (dict(V=40000, ld=40000, ws=None), _lib.GRPO_ERR_WORKSPACE), (dict(V=40000, ld=40000, ws_bytes=64), _lib.GRPO_ERR_WORKSPACE),
    (dict(V=40000, ld=40000, ws=ctypes.c_void_p(0x100008)), _lib.GRPO_ERR_ALIGN),
]


@pytest.mark.parametrize("which", ["sample", "logp"])
@pytest.mark.parametrize("kw,status", BAD_SAMPLE)
def test_sampling_refusals(lib, which, kw, status):
    assert sample(lib, which, **kw) == status


def test_sampling_refusals_of_one_entry(lib):
    assert sample(lib, "sample", u=None) == _lib.GRPO_ERR_ARG
    assert sample(lib, "sample", u=ODD) == _lib.GRPO_ERR_ALIGN
    assert sample(lib, "logp", rows=ctypes.c_void_p(0x100004)) == _lib.GRPO_ERR_ALIGN
    f = lambda T=8, V=64, ld=64, dt=1, l=D, a=D, r=D, d=D, o=D: lib.grpo_sampled_logp_bwd(l, dt, T, V, ld, a, r, d, o, None)  # noqa: E731,E741
    for kw in (dict(l=None), dict(a=None), dict(r=None), dict(d=None), dict(o=None)):
        assert f(**kw) == _lib.GRPO_ERR_ARG
    assert f(ld=60) == _lib.GRPO_ERR_SHAPE and f(T=-1) == _lib.GRPO_ERR_SHAPE and f(dt=3) == _lib.GRPO_ERR_DTYPE
    for kw in (dict(l=ODD), dict(a=ODD), dict(r=ctypes.c_void_p(0x100004)), dict(d=ODD), dict(o=ODD)):
        assert f(**kw) == _lib.GRPO_ERR_ALIGN


def test_dlogits_over_part_of_the_logits_is_refused(lib):
    """Rows of 100 columns, bf16: shifted by a column, by a row, by a column less than the row's width."""
    f = lambda d, ld, T=8: lib.grpo_sampled_logp_bwd(D, 1, T, 100, ld, D, D, D, ctypes.c_void_p(0x100000 + 2 * d), None)  # noqa: E731
    for d, ld in ((1, 100), (99, 100), (100, 100), (700, 100), (-1, 100), (-100, 100), (99, 200), (101, 200), (-99, 200),
                  (1 * 200 + 50, 200), (7 * 200 + 99, 200)):
        assert f(d, ld) == _lib.GRPO_ERR_ARG, (d, ld)


def test_sampling_workspace(lib):
    f = lib.grpo_sampling_workspace_bytes
    assert f(-1, 10) == 0 and f(1, 0) == 0 and f(1, (1 << 22) + 1) == 0
    for T, V in ((1, 151936), (100, 1 << 22), (191, 16385)):
        assert f(T, V) >= 48 * T * (V // 2048) and f(T, V) % 256 == 0
    for T, V in ((0, 1), (0, 151936), (1, 5), (191, 16384), (192, 151936), (1 << 20, 151936)):
        assert f(T, V) == 0  # none is needed


def grads(*recs):
    arr = (_lib.Grad * max(len(recs), 1))()
    for a, (data, out, n, dt, odt) in zip(arr, recs):
        a.data, a.out, a.n, a.dtype, a.out_dtype = data, out, n, dt, odt
    return arr


def table(lib, *recs, n=None, size=None):
    n = len(recs) if n is None else n
    buf = ctypes.create_string_buffer(max(lib.grpo_grad_table_bytes(n), 8) + 8)
    at = (ctypes.addressof(buf) + 7) // 8 * 8
    lay = _lib.GradLayout()
    st = lib.grpo_grad_table(grads(*recs), n, at, lib.grpo_grad_table_bytes(n) if size is None else size, ctypes.byref(lay))
    return st, lay


def test_grad_table(lib):
    A = 0x100000
    st, lay = table(lib, (A, A, 8192, 0, 0), (A + 65536, A + 65536, 8193, 1, 1), (None, None, 0, 0, 0))
    assert st == 0 and (lay.n, lay.in_place, lay.units) == (3, 1, 3)
    st, lay = table(lib, (A, A + 65536, 10, 0, 1))
    assert st == 0 and (lay.in_place, lay.units) == (0, 1)
    st, lay = table(lib)
    assert st == 0 and (lay.n, lay.in_place, lay.units) == (0, 1, 0)
    # read only: the same gradient twice counts twice
    assert table(lib, (A, A + 65536, 10, 0, 1), (A, A + 131072, 10, 0, 1))[0] == 0
    assert table(lib, (A, A + 65536, 10, 0, 1), (A + 8, A + 131072, 10, 0, 1))[0] == 0


@pytest.mark.parametrize("recs,status", [
    ([(0x1000, 0x1000, 8, 2, 0)], _lib.GRPO_ERR_DTYPE), ([(0x1000, 0x1000, 8, 0, 5)], _lib.GRPO_ERR_DTYPE),
    ([(0x1000, 0x1000, -1, 0, 0)], _lib.GRPO_ERR_SHAPE), ([(0x1000, 0x1000, 1 << 40, 0, 0)], _lib.GRPO_ERR_SHAPE),
    ([(None, 0x1000, 8, 0, 0)], _lib.GRPO_ERR_ARG), ([(0x1000, None, 8, 0, 0)], _lib.GRPO_ERR_ARG),
    ([(0x1000, 0x1000, 8, 0, 1)], _lib.GRPO_ERR_ARG),
    ([(0x1002, 0x1002, 8, 0, 0)], _lib.GRPO_ERR_ALIGN), ([(0x1000, 0x2001, 8, 1, 1)], _lib.GRPO_ERR_ALIGN),
    ([(0x1000, 0x1000, 8, 0, 0), (0x1000, 0x1000, 8, 0, 0)], _lib.GRPO_ERR_SHAPE),   # scaled twice
    ([(0x1000, 0x1000, 8, 0, 0), (0x101c, 0x101c, 8, 0, 0)], _lib.GRPO_ERR_SHAPE),   # overlap by one element
    ([(0x1000, 0x1010, 8, 0, 0)], _lib.GRPO_ERR_SHAPE),                              # out over its own data
    ([(0x1000, 0x2000, 8, 0, 0), (0x2010, 0x3000, 8, 0, 0)], _lib.GRPO_ERR_SHAPE),   # out over another's data
    ([(0x1000, 0x2000, 8, 0, 0), (0x3000, 0x2010, 8, 0, 0)], _lib.GRPO_ERR_SHAPE),   # out over another's out
    ([(0x2010, 0x3000, 800, 0, 0), (0x1000, 0x2800, 8, 0, 0)], _lib.GRPO_ERR_SHAPE),  # inside a longer range
    ([(0x1000 << i, 0x1000 << i, (1 << 40) - 1, 0, 0) for i in range(32, 52)], _lib.GRPO_ERR_SHAPE),  # too many units
])
def test_grad_table_refusals(lib, recs, status):
    assert table(lib, *recs)[0] == status


def test_grad_call_refusals(lib):
    assert table(lib, n=-1)[0] == _lib.GRPO_ERR_SHAPE and table(lib, n=(1 << 20) + 1)[0] == _lib.GRPO_ERR_SHAPE
    assert lib.grpo_grad_table_bytes(-1) == 0 and lib.grpo_grad_table_bytes((1 << 20) + 1) == 0
    assert table(lib, (0x1000, 0x1000, 8, 0, 0), size=8)[0] == _lib.GRPO_ERR_WORKSPACE
    assert lib.grpo_grad_table(None, 1, 0x1000, 1 << 20, ctypes.byref(_lib.GradLayout())) == _lib.GRPO_ERR_ARG
    _, lay = table(lib, (0x1000, 0x1000, 8, 0, 0))
    L = ctypes.byref(lay)
    assert lib.grpo_grad_sumsq(None, D, D, None) == _lib.GRPO_ERR_ARG
    assert lib.grpo_grad_sumsq(L, None, D, None) == _lib.GRPO_ERR_ARG
    assert lib.grpo_grad_sumsq(L, D, None, None) == _lib.GRPO_ERR_ARG
    assert lib.grpo_grad_sumsq(L, ctypes.c_void_p(0x100004), D, None) == _lib.GRPO_ERR_ALIGN
    assert lib.grpo_grad_clip(L, D, None, 1.0, D, None, None) == _lib.GRPO_ERR_ARG
    assert lib.grpo_grad_clip(L, D, D, -1.0, D, None, None) == _lib.GRPO_ERR_ARG
    assert lib.grpo_grad_clip(L, D, D, float("nan"), D, None, None) == _lib.GRPO_ERR_ARG
    assert lib.grpo_grad_clip(L, D, ctypes.c_void_p(0x100004), 1.0, D, None, None) == _lib.GRPO_ERR_ALIGN
    assert lib.grpo_grad_clip(L, D, D, 1.0, ODD, None, None) == _lib.GRPO_ERR_ALIGN


def test_binding_refuses_host_tensors_and_wrong_types():
    z, u = torch.zeros(3, 8), torch.zeros(3)
    a = torch.zeros(3, dtype=torch.int32)
    for call in (lambda **k: grpo.grpo_sample(z, u, **k), lambda **k: grpo.grpo_sampled_logp(z, a, **k)):
        with pytest.raises(ValueError, match="GPU"):
            call()
        with pytest.raises(TypeError):
            call(temperature=torch.ones(3, dtype=torch.float64))
        with pytest.raises(TypeError):
            call(top_k=torch.ones(3))
        with pytest.raises(ValueError):
            call(top_p=torch.ones(4))
    with pytest.raises(ValueError):
        grpo.grpo_sample(z, torch.zeros(2))
    with pytest.raises(ValueError, match="columns"):
        grpo.grpo_sample(torch.zeros(3, 16)[:, :8], u, V=9)
    with pytest.raises(TypeError):
        grpo.grpo_sample(z.half(), u)
    with pytest.raises(ValueError):
        grpo.grpo_sample(z.t(), u)
    with pytest.raises(TypeError):
        grpo.grpo_sampled_logp(z, a.long())
    with pytest.raises(TypeError):
        grpo.grpo_sampled_logp_bwd(z, a, torch.zeros(3, 32), u)
    with pytest.raises(ValueError):
        grpo.grpo_sampled_logp_bwd(z, a, torch.zeros(3, 32, dtype=torch.uint8), u, dlogits=None)
    with pytest.raises(ValueError, match="GPU"):
        grpo.GradList([z])
