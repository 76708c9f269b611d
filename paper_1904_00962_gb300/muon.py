"""Orthogonalised (Muon) update of a model's matrices on PyTorch tensors.

``MuonPlan`` holds a plan of the C library (include/lamb.h) for a list of
matrices and checks the tensors it is bound to; it does no arithmetic.  The
bound tensors are kept alive with the plan, until others take their place.
"""
from __future__ import annotations

import torch

from . import binding as B
from .state import _dtype_code, _with_index

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


class MuonPlan:
    """One step (or the direction alone) of matrices of the given shapes.
    decay_mask: 1 for each matrix that weight decay applies to."""

    def __init__(self, shapes, decay_mask=None, *, grad_dtype="f32",
                 copy_dtype=None, device="cuda:0"):
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.grad_dtype, self.copy_dtype = grad_dtype, copy_dtype
        self.device = _with_index(device)
        self._bound = {}
        if decay_mask is not None and len(decay_mask) != len(self.shapes):
            raise ValueError("decay_mask: one entry a matrix is needed")
        self.handle = B.lamb_muon_create(
            [r for r, _ in self.shapes], [c for _, c in self.shapes],
            decay_mask, _dtype_code(grad_dtype), _dtype_code(copy_dtype),
            self.device.index or 0)

    def _checked(self, name, tensors, dtype):
        tensors = list(tensors)
        if len(tensors) != len(self.shapes):
            raise ValueError(f"{name}: {len(self.shapes)} tensors are needed")
        for k, (t, shape) in enumerate(zip(tensors, self.shapes)):
            if t.dtype != dtype or tuple(t.shape) != shape or \
                    not t.is_contiguous():
                raise ValueError(f"{name}[{k}]: a contiguous {dtype} tensor "
                                 f"of shape {shape} is needed")
            if not t.is_cuda or t.get_device() != (self.device.index or 0):
                raise ValueError(f"{name}[{k}] is not on {self.device}")
        return tensors

    def _bind(self, call, stream, **lists):
        """Hands the lists' addresses to the C call.  The plan goes on with the
        tensors it had, and keeps them, unless all of it succeeds."""
        call(self.handle, *([t.data_ptr() for t in ts]
                            for ts in lists.values()),
             stream=self._stream(stream))
        self._bound.update(lists)

    def _stream(self, stream):
        """A raw stream handle: PyTorch's current one of the plan's device, or
        the given one."""
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.device.index or 0)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def bind(self, w, g, m, copy=None, stream=None):
        """The weights and momenta (fp32), gradients, and bf16 copies that
        `step` works on."""
        if (copy is not None) != (self.copy_dtype is not None):
            raise ValueError("copy: needed iff the plan has a copy_dtype")
        f32 = torch.float32
        lists = dict(w=self._checked("w", w, f32),
                     g=self._checked("g", g, _TORCH[self.grad_dtype]),
                     m=self._checked("m", m, f32))
        if copy is not None:
            lists["copy"] = self._checked("copy", copy, torch.bfloat16)
        self._bind(B.lamb_muon_bind, stream, **lists)

    def bind_direction(self, u, o, stream=None):
        """The inputs (of the gradients' type) and bf16 outputs of
        `direction`."""
        self._bind(
            B.lamb_muon_bind_direction, stream,
            u=self._checked("u", u, _TORCH[self.grad_dtype]),
            o=self._checked("o", o, torch.bfloat16))

    def step(self, hyper, d_lr: torch.Tensor, stream=None):
        """One update; d_lr: a float tensor of one element on the device."""
        if d_lr.dtype != torch.float32 or d_lr.numel() != 1 or \
                d_lr.get_device() != (self.device.index or 0):
            raise ValueError("d_lr: a float32 tensor of one element on "
                             f"{self.device} is needed")
        B.lamb_muon_step(self.handle, hyper, d_lr.data_ptr(), self._stream(stream))

    def direction(self, hyper, stream=None):
        B.lamb_muon_direction(self.handle, hyper, self._stream(stream))

    def query(self, clear=False, stream=None) -> int:
        """The plan's LAMB_STATUS_* bits (synchronises the stream)."""
        return B.lamb_muon_query(self.handle, clear, self._stream(stream))

    def destroy(self):
        if self.handle:
            B.lamb_muon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
