"""Linear layers of any width with what follows them in one call: bias, activation, dropout and a residual.

    Y = linear(X, weight, bias, activation="gelu", residual=H, p=0.1, seed=seed, offset=step)

Both directions are kernels of the library; torch supplies tensors and streams.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as pc
from .dropout import _TYPES, check_drop, counter_for, drop_struct, rows_of, used_for
from .norm import ACTIVATIONS


def linear(X: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none",
           residual: torch.Tensor | None = None, p: float = 0.0, seed=0, offset: int = 0) -> torch.Tensor:
    """``residual + dropout(activation(X @ weight.T + bias))`` of X's type: float32, bfloat16 or float16, on a GPU.

    X: (..., in), weight: (out, in) and residual: (..., out), of one type; any strides.  bias: (out,) of that type or
    float32.  activation: none, relu, silu or gelu (by erf).  p, seed, offset: see dropout; p = 0 drops nothing.
    Products of 16-bit numbers are summed in float32; those of float32 numbers are taken of three bf16 numbers each, 24 bits, and summed in
    float32 (where numbers of 2^31 and more are met, in float32 throughout, which is slow).  What follows is computed in float32 and rounded once.
    The activation's slopes are kept for the backward pass, in float32 or, for 16-bit types, as 16 bits, which are 2^-16 off at most (gelu's 2.2 2^-16, with its own arithmetic) and, of slopes below zero, 2^-10 of themselves; the gradient at
    X @ weight.T + bias, but for dropout's 1 / (1 - p), which multiplies what is summed, is rounded to X's type (in float16 infinite past 65504, which is a
    gradient of 58,000 and more where a slope is above 1; exact without an activation and with relu).
    Sums are in an order that sizes, type and how the operands lie (strides, addresses of whole 16 bytes) decide: the same bits on every run, though a
    copy that lies otherwise may give others.
    PcsrError: 2^32 rows or 2^24 columns and more, and where X, weight or the result are of more than 2^23 tiles of 64 x 64.
    There is no forward-mode derivative."""
    fast = pc.train_module()
    if fast is not None and activation in ACTIVATIONS:
        out = fast.linear(X, weight, bias, ACTIVATIONS[activation], residual, p, seed, offset)
        if out is not NotImplemented:
            return out
    if not isinstance(X, torch.Tensor) or X.dim() < 1 or X.dtype not in _TYPES or not X.is_cuda:
        raise ValueError("X must be a float32, bfloat16 or float16 CUDA tensor of one dimension or more")
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2 or weight.dtype != X.dtype or weight.device != X.device \
            or weight.shape[1] != X.shape[-1] or weight.shape[0] < 1:
        raise ValueError("weight must be (out, in) of X's type on X's GPU")
    if bias is not None and (not isinstance(bias, torch.Tensor) or bias.shape != weight.shape[:1] or bias.device != X.device
                             or bias.dtype not in (torch.float32, X.dtype)):
        raise ValueError("bias must be (out,) of float32 or X's type on X's GPU")
    if residual is not None and (not isinstance(residual, torch.Tensor) or residual.shape != (*X.shape[:-1], weight.shape[0])
                                 or residual.dtype != X.dtype or residual.device != X.device):
        raise ValueError("residual must have the result's shape and type, on X's GPU")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    p, seed, offset = check_drop(p, seed, offset, X.device)
    args = (X, weight, bias, residual)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in args) or pc.has_tangent(*args):
        return LinearFunction.apply(*args, ACTIVATIONS[activation], p, seed, offset)
    return _forward(*args, ACTIVATIONS[activation], p, seed, offset, None, False)[0]


def _check(rc, where):
    if rc != pc.PCSR_OK:
        raise pc.PcsrError(rc, where)


def _p(t):
    return None if t is None else t.data_ptr()


def _struct(x, x_stride, w, w_stride, bias, residual, r_stride, act, dtype, out, how, bias_type):
    return pc.pcsr_linear_t(x.shape[0], w.shape[1], out, _TYPES[dtype], bias_type, act, 0, x.data_ptr(), w.data_ptr(), _p(bias), _p(residual),
                            x_stride, w_stride, r_stride, how)


def _operands(X, weight):
    return *rows_of(X.detach()), *rows_of(weight.detach())


def _forward(X, weight, bias, residual, act, p, seed, offset, used, keep):
    """(Y, the activation's slopes or None)"""
    out = weight.shape[0]
    Y = torch.empty((*X.shape[:-1], out), dtype=X.dtype, device=X.device)
    x, x_stride, w, w_stride = _operands(X, weight)
    keep = keep and act != 0
    slope = torch.empty((x.shape[0], out), dtype=torch.float32 if X.dtype == torch.float32 else torch.int16, device=X.device) if keep else None
    if Y.numel() == 0:
        return Y, slope
    r, r_stride = (None, 0) if residual is None else rows_of(residual.detach())
    bias = None if bias is None else bias.detach().resolve_neg().contiguous()
    if isinstance(seed, torch.Tensor):
        seed = seed.contiguous()
    lib = pc._lib()
    a = _struct(x, x_stride, w, w_stride, bias, r, r_stride, act, X.dtype, out, drop_struct(p, seed, offset, used),
                _TYPES[X.dtype if bias is None else bias.dtype])
    need = lib.pcsr_linear_workspace(ctypes.byref(a), 0)
    ws = torch.empty(need, dtype=torch.uint8, device=X.device) if need else None
    with torch.cuda.device(X.device):
        _check(lib.pcsr_linear(ctypes.byref(a), Y.data_ptr(), _p(slope), _p(ws), torch.cuda.current_stream().cuda_stream), "pcsr_linear")
    return Y, slope


def _backward(X, weight, bias_dtype, slope, dy, act, p, seed, offset, needs):
    """(dX, dweight, dbias), None for what is not needed"""
    out = weight.shape[0]
    dx = torch.empty(X.shape, dtype=X.dtype, device=X.device) if needs[0] else None
    dw = torch.empty(weight.shape, dtype=X.dtype, device=X.device) if needs[1] else None
    db = torch.empty(out, dtype=bias_dtype, device=X.device) if needs[2] else None
    if dy.numel() == 0:
        return dx, None if dw is None else dw.zero_(), None if db is None else db.zero_()
    x, x_stride, w, w_stride = _operands(X, weight)
    g, g_stride = rows_of(dy)
    lib = pc._lib()
    a = _struct(x, x_stride, w, w_stride, None, None, 0, act, X.dtype, out, drop_struct(p, seed, offset), _TYPES[bias_dtype])
    ws = torch.empty(lib.pcsr_linear_workspace(ctypes.byref(a), 1), dtype=torch.uint8, device=X.device)
    with torch.cuda.device(X.device):
        _check(lib.pcsr_linear_backward(ctypes.byref(a), _p(slope), g.data_ptr(), g_stride, _p(dx), _p(dw), _p(db), ws.data_ptr(),
                                        torch.cuda.current_stream().cuda_stream), "pcsr_linear_backward")
    return dx, dw, db


class LinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, weight, bias, residual, act, p, seed, offset):
        used = used_for(seed, p)
        Y, slope = _forward(X, weight, bias, residual, act, p, seed, offset, used, any(ctx.needs_input_grad[:3]))
        ctx.save_for_backward(X, weight, slope, used)
        ctx.how = act, p, 0 if isinstance(seed, torch.Tensor) else seed, offset
        ctx.bias_dtype = X.dtype if bias is None else bias.dtype
        return Y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        X, weight, slope, used = ctx.saved_tensors
        act, p, seed, offset = ctx.how
        grads = None, None, None
        if any(ctx.needs_input_grad[:3]):
            grads = _backward(X, weight, ctx.bias_dtype, slope, dy, act, p, seed if used is None else used, offset, ctx.needs_input_grad[:3])
        return *grads, dy if ctx.needs_input_grad[3] else None, None, None, None, None


class Linear(torch.nn.Module):
    """linear with learned weight and bias (drawn as torch.nn.Linear draws its own).  p: dropout in training, with a counter as
    Dropout has one."""

    def __init__(self, d_in: int, d_out: int, bias: bool = True, activation: str = "none", p: float = 0.0, seed: int | None = None,
                 dtype=torch.float32, device=None):
        super().__init__()
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
        like = torch.nn.Linear(d_in, d_out, bias, device=device, dtype=dtype)
        self.weight, self.bias, self.activation = like.weight, like.bias, activation
        self.p = check_drop(p, 0, 0, None)[0]
        self.register_buffer("counter", counter_for(seed).to(device) if self.p > 0.0 else None)

    def forward(self, X, residual=None):
        if not self.training or self.p == 0.0:
            return linear(X, self.weight, self.bias, self.activation, residual)
        out = linear(X, self.weight, self.bias, self.activation, residual, self.p, self.counter)
        self.counter[1:].add_(1)
        return out

    def extra_repr(self):
        return f"{self.weight.shape[1]}, {self.weight.shape[0]}, activation={self.activation}, p={self.p}"


class FeedForward(torch.nn.Module):
    """X + dropout(W2 dropout(activation(W1 X + b1)) + b2), the block that deep graph models have behind a layer: two calls."""

    def __init__(self, width: int, hidden: int, activation: str = "gelu", p: float = 0.0, dtype=torch.float32, device=None):
        super().__init__()
        self.first = Linear(width, hidden, True, activation, p, None, dtype, device)
        self.second = Linear(hidden, width, True, "none", p, None, dtype, device)

    def forward(self, X):
        return self.second(self.first(X), residual=X)
