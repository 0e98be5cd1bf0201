"""A product with bias, activation and residual in its epilogue, and its gradient: binding of include/grpo_linear.h.

y = act(x W + bias) + residual with x [M, K] and W [K, N] in bf16.  W may be a [K, N] tensor or the transpose of an
[N, K] one (``weight.t()``), as it lies in memory: no copy is made of either unless its rows are not whole aligned vectors.
"""
from __future__ import annotations

import ctypes

import torch

from . import _check, _lib, _meta, _nbytes, _placed, _workspace
from ._lib import GRPO_BF16, GRPO_F32
from .sampling import _at, _on

ACTIVATIONS = {"none": _lib.GRPO_ACT_NONE, "relu": _lib.GRPO_ACT_RELU, "gelu": _lib.GRPO_ACT_GELU,
               "gelu_tanh": _lib.GRPO_ACT_GELU_TANH, "silu": _lib.GRPO_ACT_SILU}
_CODES = {torch.bfloat16: GRPO_BF16, torch.float32: GRPO_F32}


def _code(dtype, name):
    if dtype not in _CODES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {dtype}")
    return _CODES[dtype]


def _rows(t, name, dtype, shape=None):
    """Row stride of a 2-D tensor with unit column stride (that of a single row or column says nothing)."""
    _meta(t, name, dtype, shape=shape)
    if t.dim() != 2:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    return _row_stride(t.shape, t.stride(), name)


def _row_stride(shape, strides, name):
    (rows, cols), (ld, step) = shape, strides
    if step != 1 and cols != 1:
        raise ValueError(f"{name} must be 2-D with unit column stride")
    if rows <= 1:
        return cols
    if ld < cols:
        raise ValueError(f"{name}'s rows overlap")
    return ld


def _op(x, w, act):
    """The operator's struct without its bias."""
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    ldx = _rows(x, "x", torch.bfloat16)
    _meta(w, "w", torch.bfloat16)
    if w.dim() != 2:
        raise ValueError("w must be 2-D")
    (K, N), (s0, s1) = w.shape, w.stride()
    out_in = s1 != 1 and s0 == 1
    ldw = _row_stride((N, K), (s1, s0), "w.t()") if out_in else _row_stride((K, N), (s0, s1), "w")
    M, Kx = x.shape
    if Kx != K:
        raise ValueError(f"x and w disagree on K: {Kx} and {K}")
    return _lib.LinearOp(M, K, N, x.data_ptr(), ldx, w.data_ptr(), ldw, out_in, ACTIVATIONS[act], None, 0)


def grpo_linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None,
                residual: torch.Tensor | None = None, *, act: str = "none", out_dtype=torch.bfloat16,
                out: torch.Tensor | None = None, keep_z: bool = False, workspace: torch.Tensor | None = None,
                stream=None):
    """y = act(x w + bias) + residual: x bf16 [M, K] with unit column stride, w bf16 [K, N] with unit stride in either
    dimension, bias [N] bf16 or fp32, residual [M, N] of y's type, act "none", "relu", "gelu", "gelu_tanh" or "silu".
    ``out``: y, written in place (it may be ``residual``, and otherwise shares no element with another operand; columns of one
    buffer are in order); without it a tensor of ``out_dtype`` (bf16 or fp32).  Returns
    (y, z), z = x w + bias in fp32 with ``keep_z`` (what ``grpo_linear_bwd`` takes if there is an activation), otherwise
    None."""
    op = _op(x, w, act)
    M, N, dev = op.M, op.N, x.device
    if bias is not None:
        _meta(bias, "bias", None, shape=(N,))
        op.bias, op.bias_dtype = bias.data_ptr(), _code(bias.dtype, "bias")
    dtype = out_dtype if out is None else _meta(out, "out", None).dtype
    code = _code(dtype, "out_dtype" if out is None else "out")
    ldy = N if out is None else _rows(out, "out", dtype, (M, N))
    ldr = 0 if residual is None else _rows(residual, "residual", dtype, (M, N))
    _placed(dev, strided=("x", "w", "residual", "out"), x=x, w=w, bias=bias, residual=residual, out=out)

    def call(s):
        lib, ws = _lib.load(), workspace
        need = lib.grpo_linear_workspace_bytes(ctypes.byref(op))
        if ws is not None or need:
            ws = _workspace(ws, need, dev)
        y = torch.empty((M, N), dtype=dtype, device=dev) if out is None else out
        z = torch.empty((M, N), dtype=torch.float32, device=dev) if keep_z else None
        st = lib.grpo_linear(ctypes.byref(op), _at(residual), ldr, y.data_ptr(), ldy, code, _at(z), _at(ws),
                             0 if ws is None else _nbytes(ws), s)
        _check(st, "grpo_linear")
        return y, z

    return _on(dev, stream, call)


def grpo_linear_bwd(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, z: torch.Tensor | None = None, *,
                    act: str = "none", dx=True, dw=True, dbias: torch.Tensor | None = None, accumulate_dw: bool = False,
                    workspace: torch.Tensor | None = None, stream=None):
    """The gradients of ``grpo_linear``'s y given that call's x, w and z (fp32 [M, N]; None without an activation) and the
    incoming dy [M, N] (bf16 or fp32); the residual's is dy itself.  ``dx``: True allocates a bf16 [M, K] tensor, False is
    none, a tensor is written.  ``dw``: likewise, laid out as w ([K, N], or the transpose of [N, K]), bf16 or fp32, an fp32
    one added to with ``accumulate_dw``.  ``dbias``: a tensor [N] of the bias's type to be written, or None.  What is written
    shares no element with what is read.  Returns (dx, dw, dbias), None for those not asked for."""
    op = _op(x, w, act)
    M, K, N, dev = op.M, op.K, op.N, x.device
    lddy = _rows(dy, "dy", None, (M, N))
    code = _code(dy.dtype, "dy")
    if act == "none":
        z = None
    else:
        _meta(z, "z", torch.float32, shape=(M, N))
    given = {}
    g = _lib.LinearGrads()
    if isinstance(dx, torch.Tensor):
        given["dx"] = _meta(dx, "dx", torch.bfloat16, shape=(M, K))
    if isinstance(dw, torch.Tensor):
        _meta(dw, "dw", None, shape=(K, N))
        _code(dw.dtype, "dw")
        given["dw"] = dw.t() if op.w_out_in else dw
    if accumulate_dw and (not isinstance(dw, torch.Tensor) or dw.dtype != torch.float32):
        raise ValueError("accumulate_dw needs an fp32 dw")
    if dbias is not None:
        _meta(dbias, "dbias", None, shape=(N,))
        op.bias_dtype = _code(dbias.dtype, "dbias")
    _placed(dev, strided=("x", "w", "dy"), x=x, w=w, dy=dy, z=z, dbias=dbias, **given)
    g.accumulate_dw = bool(accumulate_dw)

    def call(s):
        lib, ws = _lib.load(), workspace
        out_x = torch.empty((M, K), dtype=torch.bfloat16, device=dev) if dx is True else dx if "dx" in given else None
        out_w = given.get("dw")
        if dw is True:
            out_w = torch.empty((N, K) if op.w_out_in else (K, N), dtype=torch.bfloat16, device=dev)
        g.dx, g.dw, g.dbias = _at(out_x), _at(out_w), _at(dbias)
        if out_w is not None:
            g.dw_dtype = _CODES[out_w.dtype]
        need = lib.grpo_linear_bwd_workspace_bytes(ctypes.byref(op), dy.data_ptr(), lddy, code, ctypes.byref(g))
        if ws is not None or need:
            ws = _workspace(ws, need, dev)
        st = lib.grpo_linear_bwd(ctypes.byref(op), dy.data_ptr(), lddy, code, _at(z), ctypes.byref(g), _at(ws),
                                 0 if ws is None else _nbytes(ws), s)
        _check(st, "grpo_linear_bwd")
        return out_x, (out_w.t() if op.w_out_in and out_w is not None else out_w), dbias

    return _on(dev, stream, call)
