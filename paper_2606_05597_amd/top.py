"""What a row of logits says about a token, with its gradient: binding of include/grpo_top.h.

The log-prob of a given token, the policy's entropy and the n likeliest alternatives with their log-probs, at a
temperature that is a number for all rows or a GPU tensor [T] with one value per row.
"""
from __future__ import annotations

import torch

from . import _check, _dlogits_arg, _lib, _meta, _nbytes, _placed, _workspace
from ._lib import GRPO_TOP_MAX
from .sampling import _at, _columns, _on

TOP_ROW_BYTES = 24  # one grpo_top_row


def _alternatives(n):
    n = int(n)
    if not 0 <= n <= GRPO_TOP_MAX:
        raise ValueError(f"n must be 0 .. {GRPO_TOP_MAX}, got {n}")
    return n


def grpo_token_logp_top(logits: torch.Tensor, actions: torch.Tensor, n: int, *, temperature=None, V: int | None = None,
                        error_flags: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Log-prob of each row's given action, entropy of the row, and its ``n`` likeliest words (0 .. 64) with their
    log-probs, the lowest index first among equal ones.  Returns (logp fp32 [T], entropy fp32 [T], ids int32 [T, n],
    top_logp fp32 [T, n], rows uint8 [T, 24], what ``grpo_token_logp_top_bwd`` takes).  A row with fewer words ends in
    id -1 and log-prob -inf; a masked action's log-prob is -inf, that of an action outside [0, V) 0."""
    dt, T, V, ld = _columns(logits, V)
    n = _alternatives(n)
    _meta(actions, "actions", torch.int32, shape=(T,))
    by_row = isinstance(temperature, torch.Tensor)
    if by_row:
        _meta(temperature, "temperature", torch.float32, shape=(T,))
    _meta(error_flags, "error_flags", torch.int32, n=1, optional=True)
    dev = logits.device
    _placed(dev, strided=("logits",), logits=logits, actions=actions, error_flags=error_flags,
            temperature=temperature if by_row else None)

    def call(s):
        lib, ws = _lib.load(), workspace
        need = lib.grpo_token_logp_top_workspace_bytes(T, V, n)
        if ws is not None or need:
            ws = _workspace(ws, need, dev)
        logp = torch.empty(T, dtype=torch.float32, device=dev)
        entropy = torch.empty(T, dtype=torch.float32, device=dev)
        top_logp = torch.empty((T, n), dtype=torch.float32, device=dev)
        ids = torch.empty((T, n), dtype=torch.int32, device=dev)
        rows = torch.empty((T, TOP_ROW_BYTES), dtype=torch.uint8, device=dev)
        st = lib.grpo_token_logp_top(logits.data_ptr(), dt, T, V, ld, temperature.data_ptr() if by_row else None,
                                     1.0 if temperature is None or by_row else temperature, actions.data_ptr(), n,
                                     logp.data_ptr(), entropy.data_ptr(), ids.data_ptr(), top_logp.data_ptr(),
                                     rows.data_ptr(), _at(error_flags), _at(ws), 0 if ws is None else _nbytes(ws), s)
        _check(st, "grpo_token_logp_top")
        return logp, entropy, ids, top_logp, rows

    return _on(dev, stream, call)


def grpo_token_logp_top_bwd(logits: torch.Tensor, actions: torch.Tensor, ids: torch.Tensor, rows: torch.Tensor,
                            dlogp: torch.Tensor | None = None, dentropy: torch.Tensor | None = None,
                            dtop: torch.Tensor | None = None, *, V: int | None = None, dlogits=True,
                            stream=None) -> torch.Tensor:
    """The gradient of ``grpo_token_logp_top``'s log-probs, entropies and alternatives' log-probs with respect to the
    logits, given that call's ``ids`` and ``rows`` and the incoming gradients (fp32 [T], [T], [T, n]; None: none).
    ``dlogits``: True allocates a tensor like ``logits``; a tensor is written in place (it may be ``logits`` itself).
    Columns past V are not written."""
    dt, T, V, ld = _columns(logits, V)
    _meta(actions, "actions", torch.int32, shape=(T,))
    _meta(ids, "ids", torch.int32)
    if ids.dim() != 2 or ids.shape[0] != T:
        raise ValueError(f"ids must be [{T}, n], got {tuple(ids.shape)}")
    n = _alternatives(ids.shape[1])
    _meta(rows, "rows", torch.uint8, shape=(T, TOP_ROW_BYTES))
    f32 = torch.float32
    _meta(dlogp, "dlogp", f32, shape=(T,), optional=True)
    _meta(dentropy, "dentropy", f32, shape=(T,), optional=True)
    _meta(dtop, "dtop", f32, shape=(T, n), optional=True)
    if dlogits is None or dlogits is False:
        raise ValueError("dlogits must be True or a tensor")
    if dlogits is not True:
        _dlogits_arg(dlogits, logits)
    dev = logits.device
    _placed(dev, strided=("logits", "dlogits"), logits=logits, dlogits=None if dlogits is True else dlogits,
            actions=actions, ids=ids, rows=rows, dlogp=dlogp, dentropy=dentropy, dtop=dtop)

    def call(s):
        out = _dlogits_arg(dlogits, logits)
        st = _lib.load().grpo_token_logp_top_bwd(logits.data_ptr(), dt, T, V, ld, actions.data_ptr(), n, ids.data_ptr(),
                                                 rows.data_ptr(), _at(dlogp), _at(dentropy), _at(dtop), out.data_ptr(), s)
        _check(st, "grpo_token_logp_top_bwd")
        return out

    return _on(dev, stream, call)
