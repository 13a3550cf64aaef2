"""Rows of a learned table by id, scaled, with the table's gradient: the input of a model whose
nodes come without features, or whose batches are samples of them.

    table = torch.nn.Parameter(torch.randn(n_nodes, d, device="cuda"))
    H = embedding(ids, table, scale=d ** 0.5)      # (*ids.shape, d)

Both directions are kernels of the library; torch supplies tensors and streams.
"""
from __future__ import annotations

import torch

from . import binding as pc

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def embedding(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """``scale * table[ids]`` of the table's type (float32, bfloat16 or float16), each number rounded once.

    ids: int32 or int64 tensor of any shape on the table's GPU.  An id outside ``[0, len(table))`` stands
    for no row (padding): zeros, and no gradient.  table: (rows, d); rows may lie apart, numbers of a
    row may not (such a table is copied).  The gradient is dense, of the table's type; its sums are
    taken in 32 bits, in an order that ids, sizes and type alone decide: the same bits on every run.  There is no forward-mode derivative."""
    fast = pc.train_module()
    if fast is not None:
        out = fast.embed(ids, table, scale)
        if out is not NotImplemented:
            return out
    if not isinstance(ids, torch.Tensor) or ids.dtype not in (torch.int32, torch.int64):
        raise ValueError("ids must be an int32 or int64 tensor")
    if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.dtype not in _TYPES or table.shape[1] < 1:
        raise ValueError("table must be a 2-D float32, bfloat16 or float16 tensor of at least one column")
    if not table.is_cuda or ids.device != table.device:
        raise ValueError("ids and table must be on one GPU")
    if table.requires_grad and torch.is_grad_enabled() or pc.has_tangent(table):  # the node refuses tangents
        return EmbeddingFunction.apply(ids, table, float(scale))
    return _lookup(ids, table, float(scale))


def _check(rc, where):
    if rc != pc.PCSR_OK:
        raise pc.PcsrError(rc, where)


def _rows_of(t):
    """The tensor, or a copy whose rows are whole, and the distance of its rows."""
    t = t.resolve_neg()
    if t.stride(1) != 1 and t.shape[1] > 1 or t.stride(0) < t.shape[1] and t.shape[0] > 1:
        t = t.contiguous()
    return t, max(t.stride(0), t.shape[1]) if t.shape[0] > 1 else t.shape[1]


def _lookup(ids, table, scale):
    ids = ids.contiguous()
    table, stride = _rows_of(table.detach())
    out = torch.empty((*ids.shape, table.shape[1]), dtype=table.dtype, device=table.device)
    with torch.cuda.device(table.device):
        _check(pc._lib().pcsr_embed(ids.numel(), table.shape[0], table.shape[1], _TYPES[table.dtype], ids.data_ptr(),
                                    ids.dtype == torch.int64, table.data_ptr(), stride, scale, out.data_ptr(),
                                    torch.cuda.current_stream().cuda_stream), "pcsr_embed")
    return out


def _gradient(ids, dout, shape, dtype, scale):
    (rows, d), n, lib = shape, ids.numel(), pc._lib()
    ids = ids.contiguous()
    dout, stride = _rows_of(dout.reshape(n, d))
    grad = torch.empty(shape, dtype=dtype, device=dout.device)
    ws = torch.empty(lib.pcsr_embed_workspace(n, rows, d), dtype=torch.uint8, device=dout.device)
    with torch.cuda.device(dout.device):
        _check(lib.pcsr_embed_backward(n, rows, d, _TYPES[dtype], ids.data_ptr(), ids.dtype == torch.int64, dout.data_ptr(),
                                       stride, scale, grad.data_ptr(), ws.data_ptr(),
                                       torch.cuda.current_stream().cuda_stream), "pcsr_embed_backward")
    return grad


class EmbeddingFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale):
        ctx.save_for_backward(ids)
        ctx.scale, ctx.shape, ctx.dtype = scale, table.shape, table.dtype
        return _lookup(ids, table, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        return None, _gradient(ids, dout, ctx.shape, ctx.dtype, ctx.scale), None


class NodeEmbedding(torch.nn.Module):
    """A table of ``n_nodes`` learned rows of ``d`` features, normal with deviation 1 / sqrt(d), and their
    lookup times ``scale``."""

    def __init__(self, n_nodes: int, d: int, scale: float = 1.0, dtype=torch.float32, device=None):
        super().__init__()
        self.scale = float(scale)
        self.weight = torch.nn.Parameter(torch.randn(n_nodes, d, dtype=dtype, device=device) * d ** -0.5)

    def forward(self, ids):
        return embedding(ids, self.weight, self.scale)
