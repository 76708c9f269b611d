"""Word table and vocabulary head of a language model on PyTorch tensors.

``VocabPlan`` holds a vocabulary plan of the C library (include/lamb.h) and
checks, before every call, that the tensors are what the call takes: type,
shape, device and contiguous rows.  It does no arithmetic; the kernels run on
PyTorch's current stream unless one is given.  A result that the plan allocates
belongs to the stream that writes it, as if it were made under
``torch.cuda.stream``: another stream that uses it waits for that one first, and
tells the allocator of its own use (``Tensor.record_stream``).
"""
from __future__ import annotations

import contextlib

import torch

from . import binding as B
from .state import _with_index

_BF16 = {torch.bfloat16: B.LAMB_BF16}
_BOTH = {torch.float32: B.LAMB_F32, torch.bfloat16: B.LAMB_BF16}


class VocabPlan:
    """Lookup, its gradient and the head's loss for a table of `vocab` rows of
    `width` columns, for up to `max_tokens` tokens a call."""

    def __init__(self, vocab, width, max_tokens, *, device="cuda:0"):
        self.device = _with_index(device)
        self.vocab, self.width = int(vocab), int(width)
        self.max_tokens = int(max_tokens)
        self._index = self.device.index or 0
        self.handle = B.lamb_vocab_create(vocab, width, max_tokens,
                                          self._index)

    # -- checks ---------------------------------------------------------------
    def _matrix(self, name, t, rows, dtypes):
        """(address, dtype code, row stride) of a [rows, width] tensor."""
        code = dtypes.get(t.dtype)
        if code is None:
            raise ValueError(f"{name}: {t.dtype} is not one of "
                             f"{list(dtypes)}")
        width = self.width
        if t.shape != (rows, width):
            raise ValueError(f"{name}: shape {tuple(t.shape)} is not "
                             f"({rows}, {width})")
        stride, step = t.stride()
        if rows <= 1:
            stride = max(stride, width)
        if (width > 1 and step != 1) or stride < width:
            raise ValueError(f"{name}: rows have to be contiguous")
        if t.get_device() != self._index:
            raise ValueError(f"{name} is not on {self.device}")
        return t.data_ptr(), code, stride

    def _vector(self, name, t, n, dtype):
        if t.dtype != dtype or t.shape != (n,) or \
                (n > 1 and t.stride(0) != 1):
            raise ValueError(f"{name}: a contiguous {dtype} tensor of {n} "
                             f"elements is needed")
        if t.get_device() != self._index:
            raise ValueError(f"{name} is not on {self.device}")
        return t.data_ptr()

    def _scalar(self, name, t):
        """A float tensor of one element, of no dimension or one."""
        return self._vector(name, t.reshape(1) if t.dim() == 0 else t, 1,
                            torch.float32)

    def _stream(self, stream):
        """A raw stream handle: PyTorch's current one of the plan's device, or
        the given one."""
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def _allocating(self, stream):
        """A context whose new tensors' memory goes on in the order of `stream`
        (the current one: None)."""
        if stream is None:
            return contextlib.nullcontext()
        if isinstance(stream, int):
            # (0 and 1 are CUDA's names of the default stream)
            stream = torch.cuda.default_stream(self.device) if stream < 2 else \
                torch.cuda.ExternalStream(stream, device=self.device)
        return torch.cuda.stream(stream)

    def _tokens(self, name, t):
        if t.dim() != 1:
            raise ValueError(f"{name}: one dimension is needed")
        return t.shape[0]

    # -- word table -----------------------------------------------------------
    def embed(self, table, ids, *, scale=1.0, out=None, dtype=None,
              stream=None):
        """scale * table[ids]: [tokens, width] in `dtype` (the table's), into
        `out` if it is given.  Ids below 0 give rows of zeros."""
        n = self._tokens("ids", ids)
        if out is None:
            with self._allocating(stream):
                out = torch.empty((n, self.width), dtype=dtype or table.dtype,
                                  device=self.device)
        B.lamb_vocab_embed(
            self.handle, *self._matrix("table", table, self.vocab, _BOTH),
            self._vector("ids", ids, n, torch.int64), n, scale,
            *self._matrix("out", out, n, _BOTH), self._stream(stream))
        return out

    def embed_grad(self, grad_out, ids, table_grad, *, scale=1.0,
                   accumulate=False, stream=None):
        """The lookup's gradient into `table_grad` (added to it with
        `accumulate`)."""
        n = self._tokens("ids", ids)
        B.lamb_vocab_embed_grad(
            self.handle, *self._matrix("grad_out", grad_out, n, _BOTH),
            self._vector("ids", ids, n, torch.int64), n, scale,
            *self._matrix("table_grad", table_grad, self.vocab, _BOTH),
            int(accumulate), self._stream(stream))
        return table_grad

    # -- vocabulary head --------------------------------------------------------
    def _head(self, hidden, weight, labels, token_loss, loss, stream):
        n = self._tokens("labels", labels)
        if loss is None:
            with self._allocating(stream):
                loss = torch.empty(1, dtype=torch.float32, device=self.device)
        h, _, hs = self._matrix("hidden", hidden, n, _BF16)
        w, _, ws = self._matrix("weight", weight, self.vocab, _BF16)
        y = self._vector("labels", labels, n, torch.int64)
        tl = 0 if token_loss is None else \
            self._vector("token_loss", token_loss, n, torch.float32)
        lp = self._scalar("loss", loss)
        return n, loss, (h, hs, w, ws, y, n), (tl or None, lp)

    def loss(self, hidden, weight, labels, *, token_loss=None, loss=None,
             stream=None):
        """Mean cross entropy (a float tensor of one element) of
        hidden @ weight.T against the labels; labels below 0 do not count."""
        _, loss, ins, outs = self._head(hidden, weight, labels, token_loss,
                                        loss, stream)
        B.lamb_vocab_loss(self.handle, *ins, *outs, self._stream(stream))
        return loss

    def loss_grad(self, hidden, weight, labels, grad_hidden, grad_weight, *,
                  scale=None, accumulate=False, token_loss=None, loss=None,
                  stream=None):
        """The loss, and the gradients of scale * loss: grad_hidden is written,
        grad_weight written or (`accumulate`) added to.  `scale`: None or a
        float tensor of one element."""
        n, loss, ins, outs = self._head(hidden, weight, labels, token_loss,
                                        loss, stream)
        gh, _, ghs = self._matrix("grad_hidden", grad_hidden, n, _BF16)
        gw, code, gws = self._matrix("grad_weight", grad_weight, self.vocab,
                                     _BOTH)
        sp = None if scale is None else self._scalar("scale", scale)
        B.lamb_vocab_loss_grad(self.handle, *ins, sp, *outs, gh, ghs, gw, code,
                               gws, int(accumulate), self._stream(stream))
        return loss

    def query(self, clear=False, stream=None) -> int:
        """The plan's LAMB_STATUS_* bits (synchronises the stream)."""
        return B.lamb_vocab_query(self.handle, clear, self._stream(stream))

    def destroy(self):
        if self.handle:
            B.lamb_vocab_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
