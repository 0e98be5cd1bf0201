"""grpo_linear.h as seen from the host (CPU only): symbols, refusals, workspace sizes; and the binding's own checks.

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
X, W, Y, R, Z, ODD = 0x1000000, 0x2000000, 0x3000000, 0x4000000, 0x5000000, 0x1000001
NAMES = ["grpo_linear_workspace_bytes", "grpo_linear", "grpo_linear_bwd_workspace_bytes", "grpo_linear_bwd"]
MOST = 8388352


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.SO):
        from paper_2606_05597_amd.build import build
        build()
    return _lib.load()


def test_header_and_exports(lib, tmp_path):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "grpo_linear.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"^\s*(?:int|size_t)\s+(\w+)\s*\(", src, flags=re.M))) == sorted(NAMES)
    out = subprocess.check_output(["nm", "-D", "--defined-only", _lib.SO], text=True)
    assert set(NAMES) <= {line.split()[-1] for line in out.splitlines() if " T " in line}
    c = tmp_path / "t.c"
    c.write_text('#include "grpo_linear.h"\n_Static_assert(sizeof(grpo_linear_op) == %d, "op");\n'
                 '_Static_assert(sizeof(grpo_linear_grads) == %d, "grads");\nint main(void) { return GRPO_ACT_NONE; }\n'
                 % (ctypes.sizeof(_lib.LinearOp), ctypes.sizeof(_lib.LinearGrads)))
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           "-I" + os.path.join(ROOT, "include"), "-c", str(c), "-o", str(tmp_path / "t.o")])


def an_op(**kw):
    o = _lib.LinearOp()
    o.M, o.K, o.N, o.x, o.ldx, o.w, o.ldw = 8, 64, 128, X, 64, W, 128
    for k, v in kw.items():
        setattr(o, k, v)
    return o


BAD_OP = [
    (dict(act=5), _lib.GRPO_ERR_ARG), (dict(act=-1), _lib.GRPO_ERR_ARG), (dict(w_out_in=2), _lib.GRPO_ERR_ARG),
    (dict(M=-1), _lib.GRPO_ERR_SHAPE), (dict(M=MOST + 1), _lib.GRPO_ERR_SHAPE), (dict(K=0), _lib.GRPO_ERR_SHAPE),
    (dict(K=MOST + 1, ldx=1 << 40), _lib.GRPO_ERR_SHAPE), (dict(N=0), _lib.GRPO_ERR_SHAPE),
    (dict(N=MOST + 1, ldw=1 << 40), _lib.GRPO_ERR_SHAPE), (dict(ldx=63), _lib.GRPO_ERR_SHAPE),
    (dict(ldw=127), _lib.GRPO_ERR_SHAPE), (dict(w_out_in=1, ldw=63), _lib.GRPO_ERR_SHAPE), (dict(x=None), _lib.GRPO_ERR_ARG),
    (dict(w=None), _lib.GRPO_ERR_ARG), (dict(x=ODD), _lib.GRPO_ERR_ALIGN), (dict(w=ODD), _lib.GRPO_ERR_ALIGN)]


def forward(lib, op, residual=R, ldr=128, y=Y, ldy=128, y_dtype=1, z=Z, ws=None, ws_bytes=0, no_op=False):
    return lib.grpo_linear(None if no_op else ctypes.byref(op), residual, ldr, y, ldy, y_dtype, z, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", BAD_OP + [(dict(bias=R, bias_dtype=4), _lib.GRPO_ERR_DTYPE),
                                                (dict(bias=ODD, bias_dtype=1), _lib.GRPO_ERR_ALIGN)])
def test_refused_operators(lib, kw, status):
    assert forward(lib, an_op(**kw), ws=0x100000, ws_bytes=1 << 40) == status


@pytest.mark.parametrize("kw,status", [
    (dict(no_op=True), _lib.GRPO_ERR_ARG), (dict(y=None), _lib.GRPO_ERR_ARG), (dict(ldy=127), _lib.GRPO_ERR_SHAPE),
    (dict(ldr=127), _lib.GRPO_ERR_SHAPE), (dict(y_dtype=2), _lib.GRPO_ERR_DTYPE), (dict(y=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(residual=ODD), _lib.GRPO_ERR_ALIGN), (dict(z=0x1000002), _lib.GRPO_ERR_ALIGN),
    (dict(residual=Y, ldr=136), _lib.GRPO_ERR_ARG)])
def test_refused_forward_arguments(lib, kw, status):
    assert forward(lib, an_op(), ws=0x100000, ws_bytes=1 << 40, **kw) == status


def grads(**kw):
    g = _lib.LinearGrads()
    g.dx, g.dw, g.dbias, g.dw_dtype = 0x6000000, 0x7000000, 0x8000000, 1
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def backward(lib, op, g, dy=Y, lddy=128, dy_dtype=1, z=Z, ws=0x100000, ws_bytes=1 << 40):
    return lib.grpo_linear_bwd(ctypes.byref(op), dy, lddy, dy_dtype, z, None if g is None else ctypes.byref(g), ws, ws_bytes,
                               None)


@pytest.mark.parametrize("kw,status", BAD_OP + [(dict(bias_dtype=4), _lib.GRPO_ERR_DTYPE)])
def test_refused_operators_of_the_backward_call(lib, kw, status):
    assert backward(lib, an_op(**kw), grads()) == status


@pytest.mark.parametrize("kw,gkw,status", [
    (dict(), None, _lib.GRPO_ERR_ARG), (dict(dy=None), {}, _lib.GRPO_ERR_ARG), (dict(lddy=127), {}, _lib.GRPO_ERR_SHAPE),
    (dict(dy_dtype=7), {}, _lib.GRPO_ERR_DTYPE), (dict(dy=ODD), {}, _lib.GRPO_ERR_ALIGN), (dict(z=None), {}, _lib.GRPO_ERR_ARG),
    (dict(z=0x1000002), {}, _lib.GRPO_ERR_ALIGN), (dict(), dict(dw_dtype=3), _lib.GRPO_ERR_DTYPE),
    (dict(), dict(accumulate_dw=1), _lib.GRPO_ERR_ARG), (dict(), dict(accumulate_dw=2, dw_dtype=0), _lib.GRPO_ERR_ARG),
    (dict(), dict(dx=ODD), _lib.GRPO_ERR_ALIGN), (dict(), dict(dw=ODD), _lib.GRPO_ERR_ALIGN),
    (dict(), dict(dbias=0x1000002), _lib.GRPO_ERR_ALIGN), (dict(ws=None), {}, _lib.GRPO_ERR_WORKSPACE),
    (dict(ws_bytes=16), {}, _lib.GRPO_ERR_WORKSPACE), (dict(ws=0x100008), {}, _lib.GRPO_ERR_ALIGN)])
def test_refused_backward_arguments(lib, kw, gkw, status):
    assert backward(lib, an_op(act=2), None if gkw is None else grads(**gkw), **kw) == status


def test_workspace(lib):
    f = lambda **kw: lib.grpo_linear_workspace_bytes(ctypes.byref(an_op(**kw)))  # noqa: E731
    assert lib.grpo_linear_workspace_bytes(None) == 0 and f(M=0) == 0 and f(K=0) == 0
    odd = f(M=100, K=63, ldx=63)  # x is laid out anew for the tiles
    assert odd >= 2 * 100 * 64 and odd % 256 == 0
    op, g = an_op(act=2), grads()
    b = lambda op=op, g=g, lddy=128: lib.grpo_linear_bwd_workspace_bytes(ctypes.byref(op), Y, lddy, 1, ctypes.byref(g))  # noqa: E731
    assert b() >= 2 * 8 * 128 and b() % 256 == 0 and b(lddy=12) == 0
    assert b(op=an_op(act=0), g=grads(dx=None, dw=None, dbias=None)) == 0


def test_binding_refusals():
    bf, f = torch.bfloat16, grpo.grpo_linear
    x, w = torch.zeros((4, 32), dtype=bf), torch.zeros((32, 16), dtype=bf)
    with pytest.raises(ValueError, match="GPU"):
        f(x, w)
    with pytest.raises(TypeError, match="x must be"):
        f(x.float(), w)
    with pytest.raises(TypeError, match="w must be"):
        f(x, w.float())
    with pytest.raises(ValueError, match="disagree"):
        f(x, w[:31])
    with pytest.raises(ValueError, match="unit column stride"):
        f(x.t().contiguous().t(), w)
    with pytest.raises(ValueError, match="act must be"):
        f(x, w, act="tanh")
    with pytest.raises(ValueError, match="bias"):
        f(x, w, torch.zeros(15))
    with pytest.raises(TypeError, match="bias"):
        f(x, w, torch.zeros(16, dtype=torch.float64))
    with pytest.raises(TypeError, match="residual"):
        f(x, w, None, torch.zeros(4, 16))
    with pytest.raises(ValueError, match="residual"):
        f(x, w, None, torch.zeros((4, 15), dtype=bf))
    with pytest.raises(TypeError, match="out_dtype"):
        f(x, w, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="out must have"):
        f(x, w, out=torch.zeros((3, 16), dtype=bf))
    with pytest.raises(ValueError, match="rows overlap"):
        f(torch.zeros(64, dtype=bf).as_strided((4, 32), (8, 1)), w)
    g, dy = grpo.grpo_linear_bwd, torch.zeros((4, 16), dtype=bf)
    with pytest.raises(ValueError, match="GPU"):
        g(dy, x, w)
    with pytest.raises(ValueError, match="dy"):
        g(dy[:3], x, w)
    with pytest.raises(ValueError, match="z is required"):
        g(dy, x, w, act="silu")
    with pytest.raises(ValueError, match="accumulate_dw"):
        g(dy, x, w, accumulate_dw=True)
    with pytest.raises(ValueError, match="accumulate_dw"):
        g(dy, x, w, dw=torch.zeros((32, 16), dtype=bf), accumulate_dw=True)
    with pytest.raises(ValueError, match="dbias"):
        g(dy, x, w, dbias=torch.zeros(4))
    with pytest.raises(ValueError, match="dx"):
        g(dy, x, w, dx=torch.zeros((4, 31), dtype=bf))
