"""Embedding of tokens (include/tkef.h, "Embedding of tokens"): scaled rows of a
table, and the table's gradient, dense (the buffer that SparsifyPlan is bound to) or as
the list that a worker sends (what UpdatePlan takes). This module only marshals
arguments; the computation runs in the library's HIP kernels.

    ep = EmbedPlan(tokens, vocab, width, dtype=torch.float32, out_dtype=torch.bfloat16, scale=s)
    x = ep.forward(table, tokens)                      # or .lookup() under autograd
    ep.backward(tokens, dx, grad_out=grad)             # the table's gradient
    ep.backward(tokens, dx, add=grad, grad_out=grad)   # added to the readout's (tied weights)
    idx, val, nnz = ep.lists(tokens, dx, offset=o)     # one worker's list

A call's tensors are all on one GPU, that of the stream it runs on; every call can be
captured into a graph, with a workspace of its own in the graph's memory. Host threads may
share a plan: its calls take turns.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import _check, _raise_on_status, _val_format, lib
from .rows import _check_vector, _dtype_code, _launch_on, _on, _out, _ptr, _RowPlan

EMBED_MAX_ROWS = 1 << 20
EMBED_MAX_WIDTH = 1 << 16


class EmbedPlan(_RowPlan):
    """Lookup of tokens (int32, any shape, contiguous; -1: padding, a row of zeros) in a
    table (vocab, width) (tkef_embed_forward), and the table's gradient
    (tkef_embed_backward, tkef_embed_lists). Results are the same on every run."""

    _destroy = "tkef_embed_plan_destroy"

    def __init__(self, rows: int, vocab: int, width: int, dtype=torch.float32, out_dtype=None,
                 grad_dtype=None, val_dtype=torch.float32, scale: float = 1.0,
                 check: bool = False):
        """rows: the most tokens a call gives. dtype: of the table; out_dtype: of the looked
        up rows and their gradient (default: the table's); grad_dtype: of the table's
        gradient (default: the table's); val_dtype: of the lists' values."""
        super().__init__(rows, vocab, dtype, 1.0, check)
        self.width, self.scale = int(width), float(scale)
        self.out_dtype = dtype if out_dtype is None else out_dtype
        self.grad_dtype = dtype if grad_dtype is None else grad_dtype
        self.val_dtype = val_dtype
        _check("tkef_embed_plan_create", lib().tkef_embed_plan_create(
            self.rows, self.vocab, self.width, _dtype_code(dtype), _dtype_code(self.out_dtype),
            _dtype_code(self.grad_dtype), _val_format(val_dtype), self.scale,
            ctypes.byref(self._h)))
        self._info("tkef_embed_plan_info")
        L = lib()
        self._forward, self._backward, self._lists = (
            L.tkef_embed_forward, L.tkef_embed_backward, L.tkef_embed_lists)

    def _tokens(self, tokens: torch.Tensor, gpu: int) -> int:
        n = tokens.numel()
        if n > self.rows:
            raise ValueError(f"tokens: the plan takes up to {self.rows}")
        _check_vector(tokens, n, torch.int32, "tokens", gpu)
        return n

    def _block(self, x: torch.Tensor, rows: int, dtype, dev, what: str) -> int:
        """Row stride of a block of `rows` rows, each contiguous."""
        if x.dim() != 2 or x.dtype != dtype or x.device != dev or not x.is_cuda:
            raise ValueError(f"{what}: expected a 2-D tensor of {dtype} on {dev}")
        if x.shape[0] != rows or x.shape[1] != self.width:
            raise ValueError(f"{what}: expected {rows} rows of {self.width}")
        if self.width > 1 and x.stride(1) != 1:
            raise ValueError(f"{what}: the elements of a row must be contiguous")
        return x.stride(0) if rows > 1 else self.width

    def forward(self, table: torch.Tensor, tokens: torch.Tensor,
                out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
        """Returns the scaled rows (n, width) of out_dtype, n = tokens.numel()."""
        dev = table.device
        ld = self._block(table, self.vocab, self.dtype, dev, "table")
        n = self._tokens(tokens, dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            if out is None:
                out, old = _out(None, (n, self.width), self.out_dtype, dev, "out"), self.width
            else:
                old = self._block(out, n, self.out_dtype, dev, "out")
            status, own = self._status_of(status, dev)
        rc = self._forward(self._h, table.data_ptr(), ld, tokens.data_ptr(), n, out.data_ptr(), old,
                           _ptr(status), h)
        if rc:
            _check("tkef_embed_forward", rc)
        if own:
            _raise_on_status("tkef_embed_forward", status, stream)
        return out

    def backward(self, tokens: torch.Tensor, dout: torch.Tensor,
                 add: Optional[torch.Tensor] = None, grad_out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The table's gradient (vocab, width) of grad_dtype from that of the rows (n, width):
        whole, with zeros for words that do not occur, or added to `add`. With grad_out=add
        only rows of words that occur are touched."""
        dev = dout.device
        n = self._tokens(tokens, dev.index)
        old = self._block(dout, n, self.out_dtype, dev, "dout")
        ald = 0 if add is None else self._block(add, self.vocab, self.grad_dtype, dev, "add")
        h = _launch_on(dev.index, stream)
        with _on(stream):
            if grad_out is None:
                grad_out = _out(None, (self.vocab, self.width), self.grad_dtype, dev, "grad_out")
                gld = self.width
            else:
                gld = self._block(grad_out, self.vocab, self.grad_dtype, dev, "grad_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._backward(
                    self._h, tokens.data_ptr(), n, dout.data_ptr(), old, _ptr(add), ald,
                    grad_out.data_ptr(), gld, _ptr(ws), self.ws_bytes, _ptr(status), h)
        if rc:
            _check("tkef_embed_backward", rc)
        if own:
            _raise_on_status("tkef_embed_backward", status, stream)
        return grad_out

    def most(self, n: int) -> int:
        """Entries that a list of n tokens may have."""
        return min(int(n), self.vocab) * self.width

    def lists(self, tokens: torch.Tensor, dout: torch.Tensor, offset: int = 0,
              idx_out: Optional[torch.Tensor] = None, val_out: Optional[torch.Tensor] = None,
              nnz_out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
              stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """The same gradient as one worker's list: positions offset + word * width + column
        (int32, ascending), their values (val_dtype), and how many there are (one int32 value
        on the GPU). Buffers that are given hold at least `most(n)` entries; those behind
        the list's end stay as they were."""
        dev = dout.device
        n = self._tokens(tokens, dev.index)
        old = self._block(dout, n, self.out_dtype, dev, "dout")
        most = self.most(n)
        for t, dtype, what in ((idx_out, torch.int32, "idx_out"), (val_out, self.val_dtype, "val_out")):
            if t is not None:
                if t.numel() < most:
                    raise ValueError(f"{what}: a list of {n} tokens has up to {most} entries")
                _check_vector(t, t.numel(), dtype, what, dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            if idx_out is None:
                idx_out = _out(None, (most,), torch.int32, dev, "idx_out")
            if val_out is None:
                val_out = _out(None, (most,), self.val_dtype, dev, "val_out")
            nnz_out = _out(nnz_out, (1,), torch.int32, dev, "nnz_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._lists(
                    self._h, tokens.data_ptr(), n, dout.data_ptr(), old, int(offset),
                    idx_out.data_ptr(), val_out.data_ptr(), nnz_out.data_ptr(), _ptr(ws),
                    self.ws_bytes, _ptr(status), h)
        if rc:
            _check("tkef_embed_lists", rc)
        if own:
            _raise_on_status("tkef_embed_lists", status, stream)
        return idx_out, val_out, nnz_out

    def lookup(self, table: torch.Tensor, tokens: torch.Tensor) -> torch.Tensor:
        """The scaled rows (n, width) as a node of torch's autograd graph, whose backward
        pass is `backward` (the table's dense gradient). grad_dtype has to be the table's.
        (A training step that is captured into a graph: torch keeps a leaf's accumulation on
        the stream of the first graph that it is part of, so no eager result of the same
        table may be alive when the backward pass is captured.)"""
        if self.grad_dtype != self.dtype:
            raise ValueError("lookup: a gradient under autograd has the table's type")
        return _Lookup.apply(table, self, tokens)


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, plan, tokens):
        ctx.plan = plan
        ctx.save_for_backward(tokens)
        return plan.forward(table, tokens)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        tokens, = ctx.saved_tensors
        # (rows that share memory, as a sum's gradient has them, are laid out)
        return ctx.plan.backward(tokens, dout.contiguous()), None, None


# ----------------------------------------------------------------------------
# one-shot calls: a plan, one execution, and TkefStatusError on any status bit
# (they synchronize), unless the caller gives a status word to check itself

def embed_tokens(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out_dtype=None,
                 status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scaled rows of the table: EmbedPlan.forward."""
    plan = EmbedPlan(max(1, tokens.numel()), table.shape[0], table.shape[1], table.dtype, out_dtype,
                     scale=scale, check=status is None)
    return plan.forward(table, tokens, status=status)


def embed_gradient(tokens: torch.Tensor, dout: torch.Tensor, vocab: int, scale: float = 1.0,
                   dtype=torch.float32, add: Optional[torch.Tensor] = None,
                   status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The table's gradient: EmbedPlan.backward."""
    plan = EmbedPlan(max(1, tokens.numel()), vocab, dout.shape[1], dtype, dout.dtype, scale=scale,
                     check=status is None)
    return plan.backward(tokens, dout, add=add, status=status)


def embed_lists(tokens: torch.Tensor, dout: torch.Tensor, vocab: int, scale: float = 1.0,
                val_dtype=torch.float32, offset: int = 0,
                status: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The list (idx, val) of the table's gradient, cut to its length (which waits for the
    GPU): EmbedPlan.lists."""
    plan = EmbedPlan(max(1, tokens.numel()), vocab, dout.shape[1], torch.float32, dout.dtype,
                     val_dtype=val_dtype, scale=scale, check=status is None)
    idx, val, nnz = plan.lists(tokens, dout, offset=offset, status=status)
    n = int(nnz.item())
    return idx[:n], val[:n]
