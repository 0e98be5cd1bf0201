"""The gradients' common norm and their clipping to it: binding of include/grpo_clip.h."""
from __future__ import annotations

import ctypes

import torch

from . import _check, _lib, _meta, _placed
from ._lib import GRPO_BF16, GRPO_F32, GRPO_GRAD_PARTIALS
from .sampling import _at, _on

_CODES = {torch.float32: GRPO_F32, torch.bfloat16: GRPO_BF16}


class GradList:
    """The gradients of a model as the clipping calls take them, laid out once and used at every step.

    ``grads``: fp32 or bf16 GPU tensors on one device, contiguous, of any shapes.  ``out``: where their clipped values
    go, a tensor of the same size for each (fp32 or bf16); None clips in place.  What is written may overlap nothing
    else.  The list holds on to the tensors' memory as it is now: gradients that are allocated anew at each step need a
    new list (the calls take a plain list of tensors too and make one).  Making a list copies its table to the device and
    waits for the current stream; while a graph is captured it raises, so a call in a graph takes a GradList made before.
    """

    def __init__(self, grads, out=None):
        grads = list(grads)
        outs = None if out is None else list(out)
        if outs is not None and len(outs) != len(grads):
            raise ValueError(f"out must hold a tensor for each of the {len(grads)} gradients, got {len(outs)}")
        every = [(f"grads[{i}]", t) for i, t in enumerate(grads)]
        every += [] if outs is None else [(f"out[{i}]", t) for i, t in enumerate(outs)]
        for name, t in every:
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
            if t.dtype not in _CODES:
                raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
        for i in range(len(grads) if outs is not None else 0):
            if outs[i].numel() != grads[i].numel():
                raise ValueError(f"out[{i}] must hold {grads[i].numel()} elements, got {outs[i].numel()}")
        self.device = every[0][1].device if every else torch.device("cuda", torch.cuda.current_device())
        _placed(self.device, **dict(every))
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing():  # the copy below waits, which would end the capture
                raise RuntimeError("a list of gradients cannot be made while a graph is captured: make a GradList before")
        # aliases: their memory stays, whatever becomes of the caller's tensors
        self._grads = [t.detach() for t in grads]
        self._outs = self._grads if outs is None else [t.detach() for t in outs]
        self._storages = {t.untyped_storage()._cdata: t.untyped_storage() for t in self._grads + self._outs}
        self._storages = list(self._storages.values())
        n = len(grads)
        recs = (_lib.Grad * max(n, 1))()
        for r, g, o in zip(recs, self._grads, self._outs):
            r.data, r.out, r.n = g.data_ptr(), o.data_ptr(), g.numel()
            r.dtype, r.out_dtype = _CODES[g.dtype], _CODES[o.dtype]
        lib = _lib.load()
        size = int(lib.grpo_grad_table_bytes(n))
        table = torch.zeros(max(size, 8), dtype=torch.uint8)
        self._layout = _lib.GradLayout()
        _check(lib.grpo_grad_table(recs, n, table.data_ptr(), size, ctypes.byref(self._layout)), "grpo_grad_table")
        self._places = [s.data_ptr() for s in self._storages]
        self._table = table.to(self.device)
        self._stream = torch._C._cuda_getCurrentRawStream(self.device.index)  # the stream that the table's memory belongs to
        self._c_args = ctypes.byref(self._layout), self._table.data_ptr()

    def __len__(self):
        return int(self._layout.n)

    def _args(self, s):
        """The library's arguments for a call on the raw stream s, the device's current one."""
        if s != self._stream:  # the list may go before that stream is done with its table
            self._table.record_stream(torch.cuda.current_stream(self.device))
        if [s.data_ptr() for s in self._storages] != self._places:
            raise ValueError("the memory of a tensor in the list has moved since the list was made")
        return self._c_args


def _grad_list(grads, out=None):
    if isinstance(grads, GradList):
        if out is not None:
            raise ValueError("out belongs to the GradList")
        return grads
    return GradList([grads] if isinstance(grads, torch.Tensor) else grads,
                    [out] if isinstance(out, torch.Tensor) else out)


def _partials(partials, device):
    if not isinstance(partials, torch.Tensor) or partials.dtype != torch.float64:
        raise TypeError("partials must be a float64 tensor")
    if tuple(partials.shape) != (GRPO_GRAD_PARTIALS,):
        raise ValueError(f"partials must have shape ({GRPO_GRAD_PARTIALS},), got {tuple(partials.shape)}")
    _placed(device, partials=partials)


def _flags(error_flags, device):
    _meta(error_flags, "error_flags", torch.int32, n=1, optional=True)
    _placed(device, error_flags=error_flags)


def _sumsq(grads, partials, s):
    if partials is None:
        partials = torch.empty(GRPO_GRAD_PARTIALS, dtype=torch.float64, device=grads.device)
    _check(_lib.load().grpo_grad_sumsq(*grads._args(s), partials.data_ptr(), s), "grpo_grad_sumsq")
    return partials


def _clip(grads, partials, max_norm, error_flags, s):
    norm = torch.empty((), dtype=torch.float32, device=grads.device)
    st = _lib.load().grpo_grad_clip(*grads._args(s), partials.data_ptr(), float(max_norm), norm.data_ptr(),
                                    _at(error_flags), s)
    _check(st, "grpo_grad_clip")
    return norm


def grpo_grad_sumsq(grads, *, partials: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The sum of squares of all gradients (a GradList, or tensors) as fp64 [GRPO_GRAD_PARTIALS] slots that add up to it;
    devices that hold different gradients of one model add their slots before each clips its own."""
    grads = _grad_list(grads)
    if partials is not None:
        _partials(partials, grads.device)
    return _on(grads.device, stream, lambda s: _sumsq(grads, partials, s))


def grpo_grad_clip(grads, partials: torch.Tensor, max_norm: float, *, out=None,
                   error_flags: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Every gradient times min(1, max_norm / (norm + 1e-6)), the norm from ``partials`` (``grpo_grad_sumsq``'s), in place
    or into the list's ``out``.  A norm that is not finite scales nothing (``error_flags``, int32 [1], then receives
    GRPO_FLAG_NONFINITE).  Returns the norm, a 0-dim fp32 tensor."""
    grads = _grad_list(grads, out)
    _partials(partials, grads.device)
    _flags(error_flags, grads.device)
    return _on(grads.device, stream, lambda s: _clip(grads, partials, max_norm, error_flags, s))


def grpo_clip_grad_norm_(grads, max_norm: float, *, out=None, error_flags: torch.Tensor | None = None,
                         stream=None) -> torch.Tensor:
    """The gradients' common norm, and the gradients clipped to ``max_norm``: ``grpo_grad_sumsq``, then
    ``grpo_grad_clip``.  Returns the norm, a 0-dim fp32 tensor.  With a GradList nothing waits for the device; a plain list
    of tensors is made into one first, which waits for the current stream."""
    grads = _grad_list(grads, out)
    _flags(error_flags, grads.device)
    return _on(grads.device, stream, lambda s: _clip(grads, _sumsq(grads, None, s), max_norm, error_flags, s))
