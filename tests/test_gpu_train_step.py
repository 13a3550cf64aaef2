"""The parts around the layers in one training step: a table of node features, norms over the graphs of a batch between the
layers, orthogonalised updates; against the same step in 64 bits on a dense adjacency."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _batch(rng, sizes):
    """Block-diagonal symmetric graph: CSR arrays, dense, offsets"""
    n = sum(sizes)
    A = np.zeros((n, n), np.float32)
    at = 0
    for k in sizes:
        m = np.triu(rng.random((k, k)) < 0.3, 1) * rng.uniform(0.2, 1.0, (k, k))
        A[at:at + k, at:at + k] = m + m.T
        at += k
    rows, cols = np.nonzero(A)
    rowptr = np.zeros(n + 1, np.int32)
    rowptr[1:] = np.cumsum(np.bincount(rows, minlength=n))
    return rowptr, cols.astype(np.int32), A[rows, cols].astype(np.float32), A, np.concatenate([[0], np.cumsum(sizes)])


def _norm64(H, off, groups, w, b):
    out = []
    for s, e in zip(off[:-1], off[1:]):
        v = H[s:e].view(e - s, groups, H.shape[1] // groups)
        if e > s:
            v = (v - v.mean((0, 2), keepdim=True)) / torch.sqrt(v.var((0, 2), unbiased=False, keepdim=True) + 1e-5)
        out.append(v.reshape(e - s, H.shape[1]))
    return torch.relu(torch.cat(out) * w + b)


@pytest.mark.parametrize("kind", ["gcn", "gin"])
def test_step_against_64_bits(kind):
    from paper_2605_15695_amd.embedding import NodeEmbedding
    from paper_2605_15695_amd.gnn import PcsrOperator, make_model
    from paper_2605_15695_amd.muon import Muon

    rng = np.random.default_rng(3)
    rowptr, colidx, vals, A, off = _batch(rng, [9, 0, 14, 1, 30])
    n = A.shape[0]
    op = PcsrOperator(n, n, rowptr, colidx, vals, symmetric=True, K_hint=16)
    torch.manual_seed(1)
    model = make_model(kind, op, 8, 16, 8, 3, norm_groups=4).cuda()
    table = NodeEmbedding(100, 8, scale=2.0, device="cuda")
    ids = torch.from_numpy(rng.integers(0, 100, n)).cuda()
    offsets = torch.from_numpy(off).cuda()
    target = torch.randn(n, 8, device="cuda")
    params = list(table.parameters()) + list(model.parameters())
    matrices = [p for p in model.parameters() if p.dim() == 2]
    opt = Muon(matrices, lr=0.05)
    start = [p.detach().double().requires_grad_() for p in params]
    loss = (model(table(ids), offsets) - target).square().mean()
    loss.backward()

    # the same in 64 bits
    A64 = torch.from_numpy(A).double().cuda()
    it = iter(start)
    H = next(it)[ids] * 2.0
    for m in model:
        name = type(m).__name__
        if name == "GroupNorm":
            H = _norm64(H, off.tolist(), 4, next(it), next(it))
        elif name == "GCNLayer":
            bias, W = next(it), next(it)
            H = A64 @ (H @ W.t()) + bias
        else:
            eps, W1, b1, W2, b2 = (next(it) for _ in range(5))
            H = torch.relu(((1 + eps) * H + A64 @ H) @ W1.t() + b1) @ W2.t() + b2
    loss64 = (H - target.double()).square().mean()
    loss64.backward()
    assert abs(float(loss.detach()) - float(loss64.detach())) < 1e-5 * float(loss64.detach())
    for p, q in zip(params, start):  # three layers of fp32 sums: 1e-4 of the gradient's size
        assert float((p.grad.double() - q.grad).norm()) <= 1e-4 * float(q.grad.norm()) + 1e-9

    opt.step()
    for p, q in zip(params, start):
        if p.dim() != 2 or not any(p is m for m in matrices):
            continue
        X = q.grad + 0.95 * q.grad
        X = X / X.norm()
        for _ in range(5):
            S = X @ X.t()
            X = 3.4445 * X + (-4.7750 * S + 2.0315 * S @ S) @ X
        want = q.detach() - 0.05 * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * X
        # gradients are 1e-4 apart, and directions of small singular values grow up to 485 times in proportion
        assert float((p.detach().double() - want).norm()) <= 0.05 * float((q.detach() - want).norm())


def test_a_model_of_them_learns():
    from paper_2605_15695_amd.embedding import NodeEmbedding
    from paper_2605_15695_amd.gnn import PcsrOperator, make_model
    from paper_2605_15695_amd.muon import Muon

    rng = np.random.default_rng(4)
    rowptr, colidx, vals, A, off = _batch(rng, [20] * 12)
    n = A.shape[0]
    op = PcsrOperator(n, n, rowptr, colidx, vals, symmetric=True, K_hint=16)
    torch.manual_seed(2)
    model = make_model("gin", op, 16, 32, 4, 3, norm_groups=4).cuda()
    table = NodeEmbedding(n, 16, scale=4.0, device="cuda")
    ids, offsets = torch.randperm(n, device="cuda"), torch.from_numpy(off).cuda()
    target = torch.randn(n, 4, device="cuda")
    matrices = [p for p in model.parameters() if p.dim() == 2]
    rest = [p for p in model.parameters() if p.dim() != 2] + list(table.parameters())
    opts = [Muon(matrices, lr=0.02), torch.optim.Adam(rest, lr=0.02)]
    losses = []
    for _ in range(80):
        for o in opts:
            o.zero_grad()
        loss = (model(table(ids), offsets) - target).square().mean()
        loss.backward()
        for o in opts:
            o.step()
        losses.append(float(loss.detach()))
    assert losses[-1] < 0.5 * losses[0], losses[::10]


def test_the_command_runs_them_together(capsys):
    import json

    from paper_2605_15695_amd import gnn_bench

    for model in ("gcn", "gin"):
        assert gnn_bench.main(["--workload", "road", "--size", "small", "--model", model, "--hidden", "32", "--steps", "3", "--warmup", "1",
                               "--embed", "--norm", "4", "--optimizer", "muon"]) == 0
        out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
        assert out["embed"] and out["norm_groups"] == 4 and out["optimizer"] == "muon" and len(out["results"]) == 1
        assert np.isfinite(out["results"][0]["final_loss"])
