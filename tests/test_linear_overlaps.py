"""Operands of the product and its gradients that share memory (CPU only): refused where a result would be written over what is
still read or over another result.  Every library call here fails host-side validation; device pointers are numbers."""
import ctypes
import os
import subprocess

import pytest

from paper_2606_05597_amd import _lib
from tests.test_linear_abi import ROOT, an_op, backward, forward, grads, lib  # noqa: F401  (lib: the fixture)

WS = dict(ws=0x100000, ws_bytes=1 << 40)


def test_the_overlap_of_rows_against_a_count_of_bytes(tmp_path):
    exe = str(tmp_path / "rows_share")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           "-I" + os.path.join(ROOT, "paper_2606_05597_amd", "csrc"),
                           os.path.join(ROOT, "tests", "rows_share.cpp"), "-o", exe])
    assert "ok" in subprocess.check_output([exe], text=True)


# x: 8 rows of 64 at 0x1000000, 128 bytes apart; w: 64 rows of 128 at 0x2000000, 256 bytes apart; y, z, residual: 8 rows of 128
@pytest.mark.parametrize("kw,op", [
    (dict(y=0x1000000), {}), (dict(y=0x10003FE), {}), (dict(y=0x1000000 - 2 * 1024 + 2), {}),  # y over x
    (dict(y=0x2000000), {}), (dict(y=0x2000000 + 2 * 64 * 128 - 2), {}),  # y over w
    (dict(y=0x2000000 + 2 * 64 * 128 - 2), dict(w_out_in=1, ldw=64)),
    (dict(residual=0x3000002), {}), (dict(residual=0x3000000 - 256), {}),  # a residual that is partly y
    (dict(residual=0x3000002, ldr=136, ldy=136), {}), (dict(residual=0x3000000 + 272, ldr=128, ldy=136), {}),
    (dict(), dict(bias=0x3000000, bias_dtype=0)), (dict(), dict(bias=0x3000000 + 2 * 1023, bias_dtype=1)),  # y over the bias
    (dict(z=0x1000000), {}), (dict(z=0x2000004), {}), (dict(z=0x3000000 - 4 * 1023), {}), (dict(z=0x4000004), {}),  # z
    (dict(), dict(bias=0x5000000, bias_dtype=0))])
def test_refused_in_the_forward_call(lib, kw, op):  # noqa: F811
    assert forward(lib, an_op(**op), **WS, **kw) == _lib.GRPO_ERR_ARG


# dy and z: 8 rows of 128 at 0x3000000 and 0x5000000; dx: 8 x 64, dw: 64 x 128, dbias: 128
@pytest.mark.parametrize("gkw,kw,act", [
    (dict(dx=0x3000000), {}, 0), (dict(dx=0x3000000 + 2 * 1023), {}, 0), (dict(dw=0x3000000 - 2 * 64 * 128 + 2), {}, 0),
    (dict(dbias=0x3000000), {}, 0), (dict(dx=0x5000000), {}, 2), (dict(dw=0x5000FFE), {}, 2), (dict(dbias=0x5000000), {}, 2),
    (dict(dx=0x1000000), {}, 0), (dict(dw=0x10003FE), {}, 0), (dict(dx=0x2000000), {}, 0),
    (dict(dw=0x6000000), {}, 0), (dict(dw=0x7000000, dbias=0x7000000), {}, 0), (dict(dbias=0x6000000), {}, 0),
    (dict(dx=0x3000000 + 250), dict(lddy=136), 0), (dict(dbias=0x3000000 + 4, dx=None, dw=None), {}, 0)])
def test_refused_in_the_backward_call(lib, gkw, kw, act):  # noqa: F811
    assert backward(lib, an_op(act=act), grads(**gkw), **kw) == _lib.GRPO_ERR_ARG
