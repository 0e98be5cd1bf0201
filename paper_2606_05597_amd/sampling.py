"""The policy as a rollout samples from it: binding of include/grpo_sampling.h.

A row's sampling distribution is its logits at a temperature, cut to the top_k likeliest words, of these to the shortest
prefix with the share top_p of their probability, of these to the words with min_p of the likeliest one's probability.
Each setting is a number for all rows or a GPU tensor [T] with one value per row.
"""
from __future__ import annotations

import ctypes

import torch

from . import _check, _dlogits_arg, _lib, _logits2d, _meta, _nbytes, _placed, _workspace
from ._lib import GRPO_SAMPLING_MAX_V

SAMPLING_ROW_BYTES = 32  # one grpo_sampling_row


def _at(t):
    return None if t is None else t.data_ptr()


def _on(device, stream, call):
    """call(the raw stream) with the tensors' device current: the caller's stream, or that device's current one.  Memory
    allocated in `call` belongs to that stream."""
    if stream is None:
        if torch._C._cuda_getDevice() == device.index:
            return call(torch._C._cuda_getCurrentRawStream(device.index))
        with torch.cuda.device(device):
            return call(torch._C._cuda_getCurrentRawStream(device.index))
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
    with torch.cuda.stream(stream):
        return call(stream.cuda_stream)


def _setting(v, name, dtype, T, tensors):
    """A setting's pointer (None where it is a number)."""
    if isinstance(v, torch.Tensor):
        _meta(v, name, dtype, shape=(T,))
        tensors[name] = v
        return v.data_ptr()
    return None


def _sampling(T, temperature, top_k, top_p, min_p):
    """The settings as a grpo_sampling struct, and the tensors among them by name."""
    tensors = {}
    f32 = torch.float32
    at = (_setting(temperature, "temperature", f32, T, tensors), _setting(top_k, "top_k", torch.int32, T, tensors),
          _setting(top_p, "top_p", f32, T, tensors), _setting(min_p, "min_p", f32, T, tensors))
    par = _lib.Sampling(*at, 1.0 if temperature is None or at[0] else temperature,
                        0 if top_k is None or at[1] else max(min(int(top_k), 2**31 - 1), 0),
                        1.0 if top_p is None or at[2] else top_p, 0.0 if min_p is None or at[3] else min_p)
    return par, tensors


def _columns(logits, V):
    dt, T, ld = _logits2d(logits)
    cols = logits.shape[1]
    V = cols if V is None else int(V)
    if V > cols:
        raise ValueError(f"V must be at most logits' {cols} columns, got {V}")
    return dt, T, V, max(ld, cols) if T == 1 else ld


def _scratch(workspace, T, V, device):
    """The caller's workspace, or a new one where the call needs one."""
    if workspace is None:
        need = _lib.load().grpo_sampling_workspace_bytes(T, V)
        if need == 0:
            return None, 0
    workspace = _workspace(workspace, 0 if workspace is not None else need, device)
    return workspace, _nbytes(workspace)


def grpo_sample(logits: torch.Tensor, u: torch.Tensor, *, temperature=None, top_k=None, top_p=None, min_p=None,
                V: int | None = None, error_flags: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None, stream=None):
    """Draws one action per row of logits [T, ld] from its sampling distribution, with the uniform random numbers ``u``
    (fp32 [T], in [0, 1)).  Settings not given are off (temperature 1).  Returns (actions int32 [T], logp fp32 [T], the
    actions' log-probs under that distribution, n_kept int32 [T], the number of words it keeps).  A row without a
    distribution (a NaN, +inf, nothing above -1e8, a setting out of range) gets action -1 and n_kept 0."""
    dt, T, V, ld = _columns(logits, V)
    _meta(u, "u", torch.float32, shape=(T,))
    par, tensors = _sampling(T, temperature, top_k, top_p, min_p)
    _meta(error_flags, "error_flags", torch.int32, n=1, optional=True)
    dev = logits.device
    _placed(dev, strided=("logits",), logits=logits, u=u, error_flags=error_flags, **tensors)

    def call(s):
        ws, ws_bytes = _scratch(workspace, T, V, dev)
        actions = torch.empty(T, dtype=torch.int32, device=dev)
        logp = torch.empty(T, dtype=torch.float32, device=dev)
        n_kept = torch.empty(T, dtype=torch.int32, device=dev)
        st = _lib.load().grpo_sample(logits.data_ptr(), dt, T, V, ld, ctypes.byref(par), u.data_ptr(),
                                     actions.data_ptr(), logp.data_ptr(), n_kept.data_ptr(), _at(error_flags), _at(ws),
                                     ws_bytes, s)
        _check(st, "grpo_sample")
        return actions, logp, n_kept

    return _on(dev, stream, call)


def grpo_sampled_logp(logits: torch.Tensor, actions: torch.Tensor, *, temperature=None, top_k=None, top_p=None,
                      min_p=None, V: int | None = None, error_flags: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, stream=None):
    """The log-prob of each row's given action under its sampling distribution.  Returns (logp fp32 [T], -inf where the
    action is not kept; n_kept int32 [T]; rows uint8 [T, 32], what ``grpo_sampled_logp_bwd`` takes)."""
    dt, T, V, ld = _columns(logits, V)
    _meta(actions, "actions", torch.int32, shape=(T,))
    par, tensors = _sampling(T, temperature, top_k, top_p, min_p)
    _meta(error_flags, "error_flags", torch.int32, n=1, optional=True)
    dev = logits.device
    _placed(dev, strided=("logits",), logits=logits, actions=actions, error_flags=error_flags, **tensors)

    def call(s):
        ws, ws_bytes = _scratch(workspace, T, V, dev)
        logp = torch.empty(T, dtype=torch.float32, device=dev)
        n_kept = torch.empty(T, dtype=torch.int32, device=dev)
        rows = torch.empty((T, SAMPLING_ROW_BYTES), dtype=torch.uint8, device=dev)
        st = _lib.load().grpo_sampled_logp(logits.data_ptr(), dt, T, V, ld, ctypes.byref(par), actions.data_ptr(),
                                           logp.data_ptr(), n_kept.data_ptr(), rows.data_ptr(), _at(error_flags),
                                           _at(ws), ws_bytes, s)
        _check(st, "grpo_sampled_logp")
        return logp, n_kept, rows

    return _on(dev, stream, call)


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
    if dlogits is not True:
        _dlogits_arg(dlogits, logits)
    dev = logits.device
    _placed(dev, strided=("logits", "dlogits"), logits=logits, dlogits=None if dlogits is True else dlogits,
            actions=actions, rows=rows, dlogp=dlogp)

    def call(s):
        out = _dlogits_arg(dlogits, logits)
        st = _lib.load().grpo_sampled_logp_bwd(logits.data_ptr(), dt, T, V, ld, actions.data_ptr(), rows.data_ptr(),
                                               dlogp.data_ptr(), out.data_ptr(), s)
        _check(st, "grpo_sampled_logp_bwd")
        return out

    return _on(dev, stream, call)
