"""Dropout and feed-forward blocks between the layers of a model, against the same step in 64 bits on a dense adjacency, and the command
that runs them."""
import json

import numpy as np
import pytest

from drop_reference import kept

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _operator(n=60):
    from paper_2605_15695_amd.gnn import PcsrOperator

    rng = np.random.default_rng(5)
    A = np.triu(rng.random((n, n)) < 0.2, 1) * rng.uniform(0.1, 0.4, (n, n))
    A = (A + A.T).astype(np.float32)
    rows, cols = np.nonzero(A)
    rowptr = np.zeros(n + 1, np.int32)
    rowptr[1:] = np.cumsum(np.bincount(rows, minlength=n))
    return PcsrOperator(n, n, rowptr, cols.astype(np.int32), A[rows, cols], symmetric=True, K_hint=16), torch.from_numpy(A).double().cuda()


def _drop64(H, p, counter):
    """counter: seed and offset, before the step"""
    if p == 0:
        return H
    k, f = kept(*H.shape, p, *counter.tolist())
    return torch.where(torch.from_numpy(k).cuda(), H * f, 0.0)


@pytest.mark.parametrize("kind", ["gcn", "gin"])
@pytest.mark.parametrize("norm,dropout,wider", [(0, 0.3, 0), (0, 0.2, 4), (4, 0.1, 3), (0, 0.0, 2)])
def test_step_against_64_bits(kind, norm, dropout, wider):
    from paper_2605_15695_amd.gnn import make_model

    op, A = _operator()
    torch.manual_seed(2)
    model = make_model(kind, op, 8, 16, 8, 3, norm, dropout, wider).cuda()
    X, target = torch.randn(60, 8, device="cuda"), torch.randn(60, 8, device="cuda")
    for step in range(2):  # the second drops others
        counters = {id(m): m.counter.clone() for m in model.modules() if getattr(m, "counter", None) is not None}
        params = [p.detach().double().requires_grad_() for p in model.parameters()]
        it = iter(params)
        H = X.double()
        for m in model:
            name = type(m).__name__
            if name == "GCNLayer":
                b, W = next(it), next(it)
                H = A @ (H @ W.t()) + b
            elif name == "GINLayer":
                eps, W1, b1, W2, b2 = (next(it) for _ in range(5))
                H = torch.relu(((1 + eps) * H + A @ H) @ W1.t() + b1) @ W2.t() + b2
            elif name == "GroupNorm":
                w, b = next(it), next(it)
                v = H.view(60, m.groups, -1)
                v = (v - v.mean((0, 2), keepdim=True)) / torch.sqrt(v.var((0, 2), unbiased=False, keepdim=True) + 1e-5)
                H = torch.relu(v.reshape(60, -1) * w + b)
            elif name == "ReLU":
                H = torch.relu(H)
            elif name == "FeedForward":
                W1, b1, W2, b2 = (next(it) for _ in range(4))
                Z = H @ W1.t() + b1
                Z = _drop64(0.5 * Z * torch.erfc(-Z / 2.0 ** 0.5), dropout, counters.get(id(m.first)))
                H = H + _drop64(Z @ W2.t() + b2, dropout, counters.get(id(m.second)))
            else:
                H = _drop64(H, dropout, counters[id(m)])
        loss64 = (H - target.double()).square().mean()
        grads64 = torch.autograd.grad(loss64, params)
        loss = (model(X) - target).square().mean()
        grads = torch.autograd.grad(loss, list(model.parameters()))
        assert abs(float(loss.detach()) - float(loss64.detach())) < 1e-5 * float(loss64.detach())
        for g, want in zip(grads, grads64):  # a few layers of fp32 sums: 1e-4 of the gradient's size
            assert float((g.double() - want).norm()) <= 1e-4 * float(want.norm()) + 1e-9
    model.eval()
    with torch.no_grad():
        assert torch.equal(model(X), model(X))


def test_the_command_runs_them(capsys):
    from paper_2605_15695_amd import gnn_bench

    for more in (["--dropout", "0.5"], ["--feed-forward", "4", "--dropout", "0.1", "--norm", "4", "--embed", "--optimizer", "muon"]):
        assert gnn_bench.main(["--workload", "road", "--size", "small", "--model", "gin", "--hidden", "32", "--steps", "3", "--warmup", "1", *more]) == 0
        out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
        assert out["dropout"] and len(out["results"]) == 1 and np.isfinite(out["results"][0]["final_loss"])
