"""Dropout of rows of features whose mask is never stored: what is dropped is a function of a seed, an offset and a number's
row and column, computed again in the backward pass.

    H = dropout(H, 0.5, seed, offset=step, residual=H_in)     # H_in + dropped H

Both directions are kernels of the library; torch supplies tensors and streams.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as pc

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_WORD = (1 << 64) - 1


def dropout(X: torch.Tensor, p: float, seed, offset: int = 0, residual: torch.Tensor | None = None) -> torch.Tensor:
    """``residual + X * kept / (1 - p)`` of X's type (float32, bfloat16 or float16, on a GPU), computed in float32 and rounded once.

    seed: an integer of up to 64 bits, and so is offset; or, for both, an int64 tensor of two numbers on X's GPU, seed and
    offset, which the kernels read when they run (a captured graph then drops others whenever they have changed; offset is not looked at).
    The backward pass uses what the forward pass did, whatever has become of that tensor.
    What is dropped: the last dimension are columns, the others rows, in order (one row, if there is one dimension).  Philox4x32-10 with the
    key seed (low word first) and the counter (column // 8, row, offset's low word, its high word) gives 16 bits to each of 8 columns, word by word, low
    half first; a number is dropped where they are below T = round(65536 p), and the others are multiplied by 65536 / (65536 - T).
    Dropped numbers count as zeros whatever they are, and so do their gradients.  X: any shape and strides, of fewer than 2^32 rows and 2^31 columns (PcsrError);
    residual: X's shape and type.  There is no forward-mode derivative."""
    fast = pc.train_module()
    if fast is not None:
        out = fast.dropout(X, p, seed, offset, residual)
        if out is not NotImplemented:
            return out
    _check_tensor(X, "X")
    if residual is not None and (not isinstance(residual, torch.Tensor) or residual.shape != X.shape or residual.dtype != X.dtype
                                 or residual.device != X.device):
        raise ValueError("residual must have X's shape and type, on X's GPU")
    p, seed, offset = check_drop(p, seed, offset, X.device)
    if torch.is_grad_enabled() and (X.requires_grad or residual is not None and residual.requires_grad) or pc.has_tangent(X, residual):
        return DropoutFunction.apply(X, residual, p, seed, offset)
    return _run(X, residual, p, seed, offset, None)


def _check_tensor(X, name):
    if not isinstance(X, torch.Tensor) or X.dim() < 1 or X.dtype not in _TYPES or not X.is_cuda:
        raise ValueError(f"{name} must be a float32, bfloat16 or float16 CUDA tensor of one dimension or more")


def check_drop(p, seed, offset, device):
    """(p, seed, offset) as the library takes them"""
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError("p must be in [0, 1]")
    if isinstance(seed, torch.Tensor):
        if seed.shape != (2,) or seed.dtype != torch.int64 or seed.device != device:
            raise ValueError("a tensor for the seed must be int64 of two numbers, seed and offset, on the rows' GPU")
        return p, seed, 0
    for v in (seed, offset):
        if not isinstance(v, int) or isinstance(v, bool) or not -(1 << 63) <= v <= _WORD:
            raise ValueError("seed and offset must be integers of 64 bits")
    return p, seed, offset


def _p(t):
    return None if t is None else t.data_ptr()


def drop_struct(p, seed, offset, used=None):
    if isinstance(seed, torch.Tensor):
        return pc.pcsr_drop_t(p, 0, 0, seed.data_ptr(), _p(used))
    return pc.pcsr_drop_t(p, seed & _WORD, offset & _WORD, None, None)


def rows_of(t):
    """(rows, columns) of a tensor, or of a copy where its rows do not lie at one distance, and that distance."""
    C, t = t.shape[-1], t.resolve_neg()
    if t.dim() != 2:
        t = t.reshape(t.shape[:-1].numel(), C)
    if t.stride(1) != 1 and C > 1 or t.stride(0) < C and t.shape[0] > 1:
        t = t.contiguous()
    return t, max(t.stride(0), C) if t.shape[0] > 1 else C


def _run(X, residual, p, seed, offset, used):
    out = torch.empty(X.shape, dtype=X.dtype, device=X.device)
    if X.numel() == 0:
        return out
    x, stride = rows_of(X.detach())
    r, r_stride = (None, 0) if residual is None else rows_of(residual.detach())
    if isinstance(seed, torch.Tensor):
        seed = seed.contiguous()
    how = drop_struct(p, seed, offset, used)
    with torch.cuda.device(X.device):
        rc = pc._lib().pcsr_dropout(*x.shape, _TYPES[X.dtype], x.data_ptr(), stride, _p(r), r_stride, ctypes.byref(how), out.data_ptr(),
                                    torch.cuda.current_stream().cuda_stream)
    if rc != pc.PCSR_OK:
        raise pc.PcsrError(rc, "pcsr_dropout")
    return out


def used_for(seed, p):
    """Where a call that reads its seed on the GPU writes what it read, for the backward pass"""
    return torch.empty(2, dtype=torch.int64, device=seed.device) if isinstance(seed, torch.Tensor) and p > 0.0 else None


class DropoutFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, residual, p, seed, offset):
        used = used_for(seed, p)
        ctx.save_for_backward(used)
        ctx.how = p, 0 if isinstance(seed, torch.Tensor) else seed, offset
        return _run(X, residual, p, seed, offset, used)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        used, = ctx.saved_tensors
        p, seed, offset = ctx.how
        dx = _run(dy, None, p, seed if used is None else used, offset, None) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


class Dropout(torch.nn.Module):
    """dropout with a seed of its own and an offset that every call in training counts up, both in ``counter``, a
    buffer: on the GPU, so that a captured graph drops others on every replay, and in the state_dict, so that a resumed training goes on with
    what comes next.  seed: an integer, or none: drawn from torch's default generator.  Copies of a module drop the same; ranks of
    a job that are seeded alike, or that are sent one rank's buffers, do too, unless they are given seeds of their own.  A forward pass that is run
    again for its activations counts on: there, call dropout with the step's own seed and offset."""

    def __init__(self, p: float = 0.5, seed: int | None = None):
        super().__init__()
        self.p = check_drop(p, 0, 0, None)[0]
        self.register_buffer("counter", counter_for(seed))

    def forward(self, X, residual=None):
        if not self.training or self.p == 0.0:
            return X if residual is None else residual + X
        out = dropout(X, self.p, self.counter, residual=residual)
        self.counter[1:].add_(1)
        return out

    def extra_repr(self):
        return f"p={self.p}"


def counter_for(seed):
    if seed is None:
        seed = int(torch.randint(0, (1 << 63) - 1, (), dtype=torch.int64))
    check_drop(0.0, seed, 0, None)
    seed &= _WORD
    return torch.tensor([seed - (1 << 64) if seed >> 63 else seed, 0], dtype=torch.int64)
