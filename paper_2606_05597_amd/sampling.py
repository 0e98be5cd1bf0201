"""The policy as a rollout samples from it: binding of include/grpo_sampling.h.

A row's sampling distribution is its logits at a temperature, cut to the top_k likeliest words, of these to the shortest
prefix with the share top_p of their probability, of these to the words with min_p of the likeliest one's probability.
Each setting is a number for all rows or a GPU tensor [T] with one value per row.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import _check, _dlogits_arg, _lib, _logits2d, _meta, _nbytes, _placed, _ptr, _workspace
from ._lib import GRPO_SAMPLING_MAX_V

SAMPLING_ROW_BYTES = 32  # one grpo_sampling_row

_SETTINGS = (("temperature", torch.float32, 1.0), ("top_k", torch.int32, 0), ("top_p", torch.float32, 1.0),
             ("min_p", torch.float32, 0.0))


@contextlib.contextmanager
def _on(device, stream):
    """The tensors' device made current and the call's raw stream on it: the caller's, or that device's current one.
    Memory allocated inside belongs to that stream."""
    if stream is not None and stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
    if stream is not None:
        with torch.cuda.stream(stream):
            yield ctypes.c_void_p(stream.cuda_stream)
    elif torch._C._cuda_getDevice() == device.index:
        yield ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(device.index))
    else:
        with torch.cuda.device(device):
            yield ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(device.index))


def _sampling(T, given):
    """The settings as a grpo_sampling struct, and the tensors among them by name."""
    par, tensors = _lib.Sampling(), {}
    for name, dtype, off in _SETTINGS:
        v = given[name]
        if isinstance(v, torch.Tensor):
            _meta(v, name, dtype, shape=(T,))
            tensors[name] = v
            setattr(par, name, v.data_ptr())
        else:
            v = off if v is None else v
            if name == "top_k":
                v = max(min(int(v), 2**31 - 1), 0)
            setattr(par, name + "_all", v)
    return par, tensors


def _columns(logits, V):
    dt, T, ld = _logits2d(logits)
    V = logits.shape[1] if V is None else int(V)
    return dt, T, V, ld


def grpo_sample(logits: torch.Tensor, u: torch.Tensor, *, temperature=None, top_k=None, top_p=None, min_p=None,
                V: int | None = None, error_flags: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None, stream=None):
    """Draws one action per row of logits [T, ld] from its sampling distribution, with the uniform random numbers ``u``
    (fp32 [T], in [0, 1)).  Settings not given are off (temperature 1).  Returns (actions int32 [T], logp fp32 [T], the
    actions' log-probs under that distribution, n_kept int32 [T], the number of words it keeps).  A row without a
    distribution (a NaN, +inf, nothing above -1e8, a setting out of range) gets action -1 and n_kept 0."""
    dt, T, V, ld = _columns(logits, V)
    _meta(u, "u", torch.float32, shape=(T,))
    par, tensors = _sampling(T, dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p))
    _meta(error_flags, "error_flags", torch.int32, n=1, optional=True)
    dev = logits.device
    _placed(dev, strided=("logits",), logits=logits, u=u, error_flags=error_flags, **tensors)
    lib = _lib.load()
    with _on(dev, stream) as s:
        workspace = _workspace(workspace, lib.grpo_sampling_workspace_bytes(T, V), dev)
        out = torch.empty((3, T), dtype=torch.int32, device=dev)
        actions, logp, n_kept = out[0], out[1].view(torch.float32), out[2]
        st = lib.grpo_sample(_ptr(logits), dt, T, V, ld, ctypes.byref(par), _ptr(u), _ptr(actions), _ptr(logp),
                             _ptr(n_kept), _ptr(error_flags), _ptr(workspace), _nbytes(workspace), s)
    _check(st, "grpo_sample")
    return actions, logp, n_kept


def grpo_sampled_logp(logits: torch.Tensor, actions: torch.Tensor, *, temperature=None, top_k=None, top_p=None,
                      min_p=None, V: int | None = None, error_flags: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, stream=None):
    """The log-prob of each row's given action under its sampling distribution.  Returns (logp fp32 [T], -inf where the
    action is not kept; n_kept int32 [T]; rows uint8 [T, 32], what ``grpo_sampled_logp_bwd`` takes)."""
    dt, T, V, ld = _columns(logits, V)
    _meta(actions, "actions", torch.int32, shape=(T,))
    par, tensors = _sampling(T, dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p))
    _meta(error_flags, "error_flags", torch.int32, n=1, optional=True)
    dev = logits.device
    _placed(dev, strided=("logits",), logits=logits, actions=actions, error_flags=error_flags, **tensors)
    lib = _lib.load()
    with _on(dev, stream) as s:
        workspace = _workspace(workspace, lib.grpo_sampling_workspace_bytes(T, V), dev)
        logp = torch.empty(T, dtype=torch.float32, device=dev)
        n_kept = torch.empty(T, dtype=torch.int32, device=dev)
        rows = torch.empty((T, SAMPLING_ROW_BYTES), dtype=torch.uint8, device=dev)
        st = lib.grpo_sampled_logp(_ptr(logits), dt, T, V, ld, ctypes.byref(par), _ptr(actions), _ptr(logp),
                                   _ptr(n_kept), _ptr(rows), _ptr(error_flags), _ptr(workspace), _nbytes(workspace), s)
    _check(st, "grpo_sampled_logp")
    return logp, n_kept, rows


def grpo_sampled_logp_bwd(logits: torch.Tensor, actions: torch.Tensor, rows: torch.Tensor, dlogp: torch.Tensor, *,
                          V: int | None = None, dlogits=True, stream=None) -> torch.Tensor:
    """The gradient of ``grpo_sampled_logp``'s log-probs with respect to the logits, given that call's ``rows`` and the
    incoming gradient ``dlogp`` (fp32 [T]).  ``dlogits``: True allocates a tensor like ``logits``; a tensor is written in
    place (it may be ``logits`` itself).  Columns past V are not written."""
    dt, T, V, ld = _columns(logits, V)
    _meta(actions, "actions", torch.int32, shape=(T,))
    _meta(rows, "rows", torch.uint8, shape=(T, SAMPLING_ROW_BYTES))
    _meta(dlogp, "dlogp", torch.float32, shape=(T,))
    if dlogits is None or dlogits is False:
        raise ValueError("dlogits must be True or a tensor")
    dlogits = _dlogits_arg(dlogits, logits) if dlogits is not True else True
    dev = logits.device
    _placed(dev, strided=("logits", "dlogits"), logits=logits, dlogits=None if dlogits is True else dlogits,
            actions=actions, rows=rows, dlogp=dlogp)
    with _on(dev, stream) as s:
        dlogits = _dlogits_arg(dlogits, logits)
        st = _lib.load().grpo_sampled_logp_bwd(_ptr(logits), dt, T, V, ld, _ptr(actions), _ptr(rows), _ptr(dlogp),
                                               _ptr(dlogits), s)
    _check(st, "grpo_sampled_logp_bwd")
    return dlogits
