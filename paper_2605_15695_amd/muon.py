"""Updates of weight matrices orthogonalised by Newton-Schulz products, and the optimiser that steps with
them (Muon: momentum, orthogonalised, per matrix).

    opt = Muon([p for p in model.parameters() if p.dim() == 2], lr=0.02)
    rest = torch.optim.Adam([p for p in model.parameters() if p.dim() != 2])

Momentum, products and the update of the weights are kernels of the library: matrices of up to 128 x 128 take one
launch for up to 24 of them, larger ones three per Newton-Schulz step for up to 24 of one shape.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch

from . import binding as pc

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
MAX_STEPS = 16
# the quintic published with the Muon optimiser (Jordan and others, 2024), which takes singular values from 0.01 to 1 to about 0.7 to 1.2 in five steps
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _coefficients(coefficients, steps):
    """ctypes array of (a, b, c) for each step"""
    if not isinstance(steps, int):  # before the look-up, to which 5 and 5.0 are the same
        raise ValueError("steps must be a whole number")
    try:
        return _coefficient_array(coefficients, steps)
    except TypeError:  # lists cannot be looked up
        return _coefficient_array.__wrapped__(coefficients, steps)


@functools.lru_cache(maxsize=64)
def _coefficient_array(coefficients, steps):
    if not 1 <= steps <= MAX_STEPS:
        raise ValueError(f"steps must be 1 to {MAX_STEPS}")
    rows = list(coefficients)
    if rows and not isinstance(rows[0], (tuple, list)):
        rows = [rows] * steps
    if len(rows) != steps or any(len(r) != 3 for r in rows):
        raise ValueError("coefficients are a triple, or one for each step")
    return (ctypes.c_double * (3 * steps))(*(float(v) for r in rows for v in r))


def _ld(t):
    """Distance of rows of a matrix whose numbers lie one behind the other, None if they do not."""
    if t.stride(1) != 1 and t.shape[1] > 1 or t.stride(0) < t.shape[1] and t.shape[0] > 1:
        return None
    return max(t.stride(0), t.shape[1]) if t.shape[0] > 1 else t.shape[1]


def _run(matrices, dtype, device, steps, coefficients, update=False, nesterov=False, momentum=0.0, keep=0.0):
    lib = pc._lib()
    how = pc.pcsr_ortho_t(_TYPES[dtype], steps, ctypes.addressof(coefficients), int(update), int(nesterov), momentum, keep)
    many = (pc.pcsr_matrix_t * len(matrices))(*matrices)
    need = lib.pcsr_ortho_workspace(many, len(matrices), ctypes.byref(how))
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    with torch.cuda.device(device):
        rc = lib.pcsr_orthogonalize(many, len(matrices), ctypes.byref(how), None if ws is None else ws.data_ptr(),
                                    torch.cuda.current_stream().cuda_stream)
    if rc != pc.PCSR_OK:
        raise pc.PcsrError(rc, "pcsr_orthogonalize")


@torch.no_grad()
def orthogonalize(G: torch.Tensor, steps: int = 5, coefficients=COEFFICIENTS) -> torch.Tensor:
    """The matrix, or each of a stack, with its singular values s taken to p(p(...(s / norm))), p(s) = a s + b s^3 + c s^5,
    `steps` times over, and its singular vectors kept; norm is the Frobenius norm, and a matrix of zeros stays one.

    G: (rows, columns) or (matrices, rows, columns) of float32, bfloat16 or float16 on a GPU; any strides.
    coefficients: (a, b, c), or one for each step.  The result has G's type; products are taken of 22 bits of their
    operands and summed in 32; X itself is held in 32.  The result is a constant to autograd, and a G that carries a
    forward-mode tangent is refused."""
    fast = pc.train_module()
    if fast is not None and isinstance(steps, int):
        co = _coefficients(coefficients, steps)
        out = fast.orthogonalize(G, steps, ctypes.addressof(co))
        if isinstance(out, int):
            raise pc.PcsrError(out, "pcsr_orthogonalize")
        if out is not NotImplemented:
            return out
    if not isinstance(G, torch.Tensor) or G.dim() not in (2, 3) or G.dtype not in _TYPES or not G.is_cuda:
        raise ValueError("G must be a float32, bfloat16 or float16 CUDA tensor of two or three dimensions")
    if pc.has_tangent(G):
        raise NotImplementedError("orthogonalize has no forward-mode derivative")
    co = _coefficients(coefficients, steps)
    out = torch.empty(G.shape, dtype=G.dtype, device=G.device)
    if G.numel() == 0:
        return out
    G = G.detach().resolve_neg()
    mats = [(G, out)] if G.dim() == 2 else list(zip(G, out))
    if _ld(mats[0][0]) is None:
        G = G.contiguous()
        mats = [(G, out)] if G.dim() == 2 else list(zip(G, out))
    rows, cols = G.shape[-2:]
    _run([pc.pcsr_matrix_t(g.data_ptr(), None, o.data_ptr(), rows, cols, _ld(g), 0, cols, 0.0, 0) for g, o in mats],
         G.dtype, G.device, steps, co)
    return out


class Muon(torch.optim.Optimizer):
    """Steps of matrices: buf = momentum * buf + grad, U = grad + momentum * buf (nesterov) or buf, and
    weight = (1 - lr * weight_decay) * weight - lr * sqrt(max(1, rows / columns)) * orthogonalize(U).

    Parameters are matrices of float32, bfloat16 or float16 on a GPU (biases, eps and tables belong to another
    optimiser); the momentum is float32."""

    def __init__(self, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 steps: int = 5, coefficients=COEFFICIENTS):
        if not lr >= 0.0 or not 0.0 <= momentum < 1.0 or not weight_decay >= 0.0:
            raise ValueError("lr and weight_decay must not be negative, momentum must be in [0, 1)")
        _coefficients(coefficients, steps)
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps,
                                      coefficients=coefficients))

    def add_param_group(self, group):
        super().add_param_group(group)
        for p in self.param_groups[-1]["params"]:
            if p.dim() != 2 or p.dtype not in _TYPES:
                self.param_groups.pop()
                raise ValueError("Muon steps matrices of float32, bfloat16 or float16")

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # torch casts state to the parameters' type and shares it with the dictionary
        for group, saved in zip(self.param_groups, state_dict["param_groups"]):
            for p, k in zip(group["params"], saved["params"]):
                if "momentum" in state_dict["state"].get(k, {}):
                    self.state[p]["momentum"] = state_dict["state"][k]["momentum"].to(p.device, torch.float32, copy=True)

    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        fast = pc.train_module()
        for group in self.param_groups:
            steps, nesterov, momentum, lr = group["steps"], group["nesterov"], float(group["momentum"]), float(group["lr"])
            keep = 1.0 - lr * float(group["weight_decay"])
            co = _coefficients(group["coefficients"], steps)
            if fast is not None:
                try:
                    bufs = [self.state[p]["momentum"] for p in group["params"]]
                except KeyError:  # the first step
                    bufs = None
                if bufs:
                    rc = fast.update(group["params"], bufs, lr, steps, ctypes.addressof(co), nesterov, momentum, keep)
                    if rc is not NotImplemented:
                        if rc != pc.PCSR_OK:
                            raise pc.PcsrError(rc, "pcsr_orthogonalize")
                        continue
            self._step_group(group, steps, nesterov, momentum, lr, keep, co)
        return loss

    @torch.no_grad()
    def _step_group(self, group, steps, nesterov, momentum, lr, keep, co):
        by_type, back = {}, []
        params = [p for p in group["params"] if p.grad is not None and p.numel()]
        for p in params:
            if not p.is_cuda or p.grad.layout != torch.strided or p.grad.dtype != p.dtype:
                raise ValueError("Muon steps dense matrices on a GPU, with gradients of their type")
            buf, grad, out = self._momentum(p), p.grad.resolve_neg(), p.detach()
            if _ld(grad) is None:
                grad = grad.contiguous()
            if _ld(out) is None or out.is_neg():
                out = out.resolve_neg().contiguous()
                back.append((p, out))
            rate = lr * math.sqrt(max(1.0, p.shape[0] / p.shape[1]))
            by_type.setdefault((p.dtype, p.device), []).append((grad, pc.pcsr_matrix_t(
                grad.data_ptr(), buf.data_ptr(), out.data_ptr(), *p.shape, _ld(grad), _ld(buf), _ld(out), rate, 0)))
        for (dtype, device), mats in by_type.items():
            _run([m for _, m in mats], dtype, device, steps, co, True, nesterov, momentum, keep)
        for p, out in back:
            p.copy_(out)
        torch.autograd.graph.increment_version(params)

    def _momentum(self, p):
        state = self.state[p]
        buf = state.get("momentum")
        if buf is None:
            buf = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
        elif buf.shape != p.shape or buf.dtype != torch.float32 or buf.device != p.device or _ld(buf) is None:
            buf = buf.to(p.device, torch.float32).reshape(p.shape).contiguous()
        state["momentum"] = buf
        return buf
