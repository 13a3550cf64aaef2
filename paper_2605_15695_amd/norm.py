"""Group norm with an activation over rows of channels (channels last), for what lies between graph
layers: nodes are rows, features are channels, and the graphs of a batch are stretches of rows.

    H = group_norm(H, 8, weight, bias, offsets=batch_offsets, activation="silu")

Both directions are kernels of the library; torch supplies tensors and streams.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as pc

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def group_norm(X: torch.Tensor, groups: int, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               offsets: torch.Tensor | None = None, eps: float = 1e-5, activation: str = "none") -> torch.Tensor:
    """``activation(xhat * weight + bias)`` of X's type, where xhat is X less its mean over the square root of its
    variance + eps, both over the rows of a graph and the channels of a group (channels / groups each).

    X: (rows, channels), one graph, or with ``offsets`` several; or (graphs, ..., channels), a graph for
    each index of the first dimension.  float32, bfloat16 or float16, on a GPU.
    offsets: int32 or int64 of (graphs + 1): graph s has the rows from offsets[s] to offsets[s + 1], so they
    ascend from 0 to the number of rows, and a graph without rows is allowed.  In host memory they are checked and
    uploaded; on the GPU they are taken as they are (the call does not wait), and offsets that do not
    ascend give wrong numbers, never an access outside the arrays.
    weight, bias: (channels,) of one type, float32 or X's.  activation: none, relu, silu or gelu (by erf,
    not tanh; below zero good to (16 + 2 z^2) 2^-24 of itself).
    A group has 2048 channels at most (4096 in 16 bits).  There are 2^22 channels at most, and 2^26 graphs, 2^24 where a graph has
    more than 8 KB on the average or a group more than 1 KB of a row (more than 4: 2^23); PcsrError otherwise.
    Statistics are float32 at least, sums in an order that sizes, offsets and type alone decide.  There is no forward-mode derivative."""
    fast = pc.train_module()
    if fast is not None and activation in ACTIVATIONS:
        out = fast.group_norm(X, groups, weight, bias, offsets, eps, ACTIVATIONS[activation])
        if out is not NotImplemented:
            return out
    if not isinstance(X, torch.Tensor) or X.dim() < 2 or X.dtype not in _TYPES or not X.is_cuda:
        raise ValueError("X must be a float32, bfloat16 or float16 CUDA tensor of two dimensions or more")
    C = X.shape[-1]
    if not isinstance(groups, int) or groups < 1 or C < 1 or C % groups:
        raise ValueError(f"{C} channels do not make {groups} groups")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    if not eps >= 0.0:
        raise ValueError("eps must not be negative")
    for p in (weight, bias):
        if p is not None and (p.shape != (C,) or p.device != X.device or p.dtype not in (torch.float32, X.dtype)):
            raise ValueError("weight and bias must be (channels,) of float32 or X's type on X's GPU")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must be of one type")
    if offsets is not None:
        offsets = _checked_offsets(offsets, X)
    args = (X, weight, bias)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in args) or pc.has_tangent(*args):  # the node refuses tangents
        return GroupNormFunction.apply(*args, groups, offsets, float(eps), ACTIVATIONS[activation])
    return _forward(*args, groups, offsets, float(eps), ACTIVATIONS[activation])[0]


def _checked_offsets(offsets, X):
    if X.dim() != 2:
        raise ValueError("offsets go with X of two dimensions")
    if not isinstance(offsets, torch.Tensor) or offsets.dtype not in (torch.int32, torch.int64) or offsets.dim() != 1:
        raise ValueError("offsets must be a 1-D int32 or int64 tensor")
    if offsets.numel() < 1 or offsets.numel() == 1 and X.shape[0]:
        raise ValueError("offsets must have an entry for each graph and one more")
    if not offsets.is_cuda:
        o = offsets.long()
        if int(o[0]) != 0 or int(o[-1]) != X.shape[0] or bool((o[1:] < o[:-1]).any()):
            raise ValueError("offsets must ascend from 0 to the number of rows")
        return offsets.to(X.device)
    if offsets.device != X.device:
        raise ValueError("offsets and X must be on one GPU")
    return offsets.contiguous()


def _check(rc, where):
    if rc != pc.PCSR_OK:
        raise pc.PcsrError(rc, where)


def _rows_of(t):
    """(rows, channels) of a tensor, or of a copy where its rows do not lie at one distance, and that distance."""
    C, t = t.shape[-1], t.resolve_neg()
    if t.dim() != 2:
        t = t.reshape(-1, C)
    if t.stride(1) != 1 and C > 1 or t.stride(0) < C and t.shape[0] > 1:
        t = t.contiguous()
    return t, max(t.stride(0), C) if t.shape[0] > 1 else C


def _p(t):
    return None if t is None else t.data_ptr()


def _struct(X, weight, bias, groups, offsets, eps, act, graphs, x, stride, mean, rstd):
    p = weight if weight is not None else bias
    return pc.pcsr_norm_t(x.shape[0], x.shape[1], groups, graphs, _p(offsets),
                          int(offsets is not None and offsets.dtype == torch.int64), _TYPES[X.dtype],
                          0 if p is None else _TYPES[p.dtype], act, x.data_ptr(), stride, _p(weight), _p(bias), eps,
                          mean.data_ptr(), rstd.data_ptr())


def _forward(X, weight, bias, groups, offsets, eps, act):
    x, stride = _rows_of(X.detach())
    graphs = offsets.numel() - 1 if offsets is not None else 1 if X.dim() == 2 else X.shape[0]
    weight, bias = (None if p is None else p.detach().resolve_neg().contiguous() for p in (weight, bias))
    stats = torch.empty((2, graphs, groups), dtype=torch.float32, device=X.device)
    y = torch.empty(X.shape, dtype=X.dtype, device=X.device)
    if x.shape[0]:
        lib = pc._lib()
        a = _struct(X, weight, bias, groups, offsets, eps, act, graphs, x, stride, stats[0], stats[1])
        ws = torch.empty(lib.pcsr_norm_workspace(ctypes.byref(a), 0), dtype=torch.uint8, device=X.device)
        with torch.cuda.device(X.device):
            _check(lib.pcsr_norm(ctypes.byref(a), y.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream),
                   "pcsr_norm")
    return y, stats, graphs


def _backward(X, weight, bias, offsets, stats, dy, groups, eps, act, graphs, needs):
    """(dX, dweight, dbias), None for what is not needed"""
    x, stride = _rows_of(X.detach())
    g, g_stride = _rows_of(dy)
    dx = torch.empty(X.shape, dtype=X.dtype, device=X.device) if needs[0] else None
    dw = torch.empty(weight.shape, dtype=weight.dtype, device=X.device) if needs[1] else None
    db = torch.empty(bias.shape, dtype=bias.dtype, device=X.device) if needs[2] else None
    if not x.shape[0]:
        return dx, None if dw is None else dw.zero_(), None if db is None else db.zero_()
    weight, bias = (None if p is None else p.detach().resolve_neg().contiguous() for p in (weight, bias))
    lib = pc._lib()
    a = _struct(X, weight, bias, groups, offsets, eps, act, graphs, x, stride, stats[0], stats[1])
    ws = torch.empty(lib.pcsr_norm_workspace(ctypes.byref(a), 1), dtype=torch.uint8, device=X.device)
    with torch.cuda.device(X.device):
        _check(lib.pcsr_norm_backward(ctypes.byref(a), g.data_ptr(), g_stride, _p(dx), _p(dw), _p(db), ws.data_ptr(),
                                      torch.cuda.current_stream().cuda_stream), "pcsr_norm_backward")
    return dx, dw, db


class GroupNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, weight, bias, groups, offsets, eps, act):
        y, stats, graphs = _forward(X, weight, bias, groups, offsets, eps, act)
        ctx.save_for_backward(X, weight, bias, offsets, stats)
        ctx.rest = groups, eps, act, graphs
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        X, weight, bias, offsets, stats = ctx.saved_tensors
        return *_backward(X, weight, bias, offsets, stats, dy, *ctx.rest, ctx.needs_input_grad[:3]), None, None, None, None


class GroupNorm(torch.nn.Module):
    """group_norm with learned weight and bias."""

    def __init__(self, groups: int, channels: int, eps: float = 1e-5, activation: str = "none"):
        super().__init__()
        if not isinstance(groups, int) or groups < 1 or channels % groups:
            raise ValueError(f"{channels} channels do not make {groups} groups")
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
        self.groups, self.eps, self.activation = groups, eps, activation
        self.weight = torch.nn.Parameter(torch.ones(channels))
        self.bias = torch.nn.Parameter(torch.zeros(channels))

    def forward(self, X, offsets=None):
        return group_norm(X, self.groups, self.weight, self.bias, offsets, self.eps, self.activation)
