"""Rows of a table by id and the table's gradient against plain torch in 64 bits.

A number of the forward pass is one product in 32 bits, rounded once: it has to be the same bits.  A gradient of
k terms is off by at most k * 2^-24 of the sum of their magnitudes (each addition, and the product with the
scale), and by half a unit in the last place of its type."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ids(g, n, rows, how):
    if how == "one":
        return torch.full((n,), rows // 2, device="cuda")
    if how == "skewed":
        return (torch.rand(n, generator=g, device="cuda", dtype=torch.float64) ** 6 * rows).long().clamp_(max=rows - 1)
    if how == "outside":  # a third of them stand for no row
        return torch.randint(-rows, 2 * rows, (n,), generator=g, device="cuda")
    return torch.randint(0, rows, (n,), generator=g, device="cuda")


def n_one(ids):
    return ids.numel() > 1 and bool((ids == ids[0]).all())


def _reference(ids, dout, rows, scale):
    ok = (ids >= 0) & (ids < rows)
    at = torch.where(ok, ids, rows).long()
    d = dout.double() * scale
    if n_one(ids):  # (adding them to one row by atomics takes a minute)
        grad, size = torch.zeros(2, rows, d.shape[1], dtype=torch.float64, device="cuda")
        if bool(ok.all()):
            grad[ids[0]], size[ids[0]] = d.sum(0), d.abs().sum(0)
        return grad, size, torch.bincount(at, minlength=rows + 1)[:rows]
    grad = torch.zeros(rows + 1, d.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, d)[:rows]
    size = torch.zeros(rows + 1, d.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, d.abs())[:rows]
    count = torch.bincount(at, minlength=rows + 1)[:rows]
    return grad, size, count


def _check(ids, table, dout, scale, kind):
    from paper_2605_15695_amd.embedding import embedding

    u = TYPES[kind][1]
    rows = table.shape[0]
    leaf = table.detach().requires_grad_()
    out = embedding(ids, leaf, scale)
    ok = ((ids >= 0) & (ids < rows)).unsqueeze(-1)
    want = torch.where(ok, (table.float()[torch.where(ok.squeeze(-1), ids, 0).long()] * scale), 0.0).to(table.dtype)
    assert out.shape == want.shape and torch.equal(out, want)
    assert torch.equal(embedding(ids, table.detach(), scale), want)
    grad, = torch.autograd.grad(out, leaf, dout)
    ref, size, count = _reference(ids.reshape(-1), dout.reshape(-1, table.shape[1]), rows, scale)
    assert grad.dtype == table.dtype and grad.shape == table.shape
    bound = size * (count.unsqueeze(1) + 1) * 2.0 ** -24 + (ref.abs() + size * 1e-3) * u + 2.0 ** -25
    assert bool(((grad.double() - ref).abs() <= bound).all())
    assert not bool(grad[count == 0].any())
    again, = torch.autograd.grad(embedding(ids, leaf, scale), leaf, dout)
    assert torch.equal(grad, again)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (64, 4), (1000, 64), (5000, 75), (70000, 33), (129, 1000), (40, 2051), (700, 20)])
@pytest.mark.parametrize("n,how", [(1, "any"), (2, "one"), (63, "any"), (65, "skewed"), (777, "outside"), (4096, "skewed"), (4097, "skewed"),
                                   (8200, "one"), (16385, "skewed"), (16384, "outside")])
def test_against_64_bits(kind, rows, d, n, how):
    g = _gen(n * 31 + rows + d)
    if n * d > 1 << 18:
        n = (1 << 18) // d
    ids = _ids(g, n, rows, how)
    table = torch.randn(rows, d, generator=g, device="cuda").to(TYPES[kind][0])
    dout = torch.randn(n, d, generator=g, device="cuda").to(TYPES[kind][0])
    _check(ids if (n + d) % 2 else ids.to(torch.int32), table, dout, 1.7, kind)


# three passes of the sort, more than one stretch of ids to a workgroup of it, runs of one id over hundreds of tiles
@pytest.mark.parametrize("n,rows,d,how", [(300_000, 1 << 20, 16, "skewed"), (1_300_000, 1 << 21, 4, "any"),
                                          (400_000, 5, 8, "any"), (200_000, 3000, 8, "one"), (100_000, 1500, 40, "outside")])
@pytest.mark.parametrize("wide", [False, True])
def test_many_ids(n, rows, d, how, wide):
    g = _gen(n + d)
    ids = _ids(g, n, rows, how).to(torch.int64 if wide else torch.int32)
    table = torch.randn(rows, d, generator=g, device="cuda")
    _check(ids, table, torch.randn(n, d, generator=g, device="cuda"), 0.5, "fp32")


def test_a_gradient_is_the_difference_of_the_function():
    from paper_2605_15695_amd.embedding import embedding

    g = _gen(2)
    table = torch.randn(9, 5, generator=g, device="cuda")
    ids = torch.tensor([[3, 3, -1], [8, 0, 3]], device="cuda")
    dout = torch.randn(2, 3, 5, generator=g, device="cuda")
    leaf = table.clone().requires_grad_()
    grad, = torch.autograd.grad(embedding(ids, leaf, 2.0), leaf, dout)

    def value(t):
        return float((embedding(ids, t, 2.0).double() * dout.double()).sum())

    for r, c in ((3, 1), (8, 0), (0, 4), (5, 2)):
        up, down = table.clone(), table.clone()
        up[r, c] += 0.5
        down[r, c] -= 0.5
        # linear: the difference is exact but for the rounding of four products of size below 10
        assert abs(value(up) - value(down) - float(grad[r, c])) < 1e-5


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_and_alignment(kind):
    dtype = TYPES[kind][0]
    g = _gen(5)
    big = torch.randn(50, 200, generator=g, device="cuda").to(dtype)
    ids = torch.randint(0, 50, (7, 100), generator=g, device="cuda")[:, ::3]
    for table in (big[:, 3:78], big[:, ::2], big[::2, 1:2], big.t()[:50, :33], big[:1].expand(50, 200)):
        flat = torch.randn(ids.numel() * 2 * table.shape[1] + 1, generator=g, device="cuda").to(dtype)
        dout = flat[1:].view(-1, 2 * table.shape[1])[:, :table.shape[1]].unflatten(0, ids.shape)
        _check(ids, table, dout, -3.0, kind)
    _check(ids, big, torch.ones(1, 1, 1, device="cuda", dtype=dtype).expand(*ids.shape, 200), 1.0, kind)


def test_infinities_and_nan_stay_in_their_rows():
    from paper_2605_15695_amd.embedding import embedding

    table = torch.ones(10, 6, device="cuda").requires_grad_()
    ids = torch.tensor([1, 2, 2, -1, 5, 10], device="cuda")
    dout = torch.ones(6, 6, device="cuda")
    dout[1, 0], dout[2, 1], dout[3] = float("inf"), float("nan"), float("nan")
    grad, = torch.autograd.grad(embedding(ids, table, 2.0), table, dout)
    want = torch.zeros(10, 6, device="cuda")
    want[1], want[5], want[2] = 2.0, 2.0, 4.0
    want[2, 0], want[2, 1] = float("inf"), float("nan")
    assert torch.equal(grad.nan_to_num(nan=-7.0), want.nan_to_num(nan=-7.0))


def test_empty_inputs():
    from paper_2605_15695_amd.embedding import embedding

    for ids_shape, rows in (((0,), 12), ((3, 0), 12), ((5,), 0)):
        table = torch.randn(rows, 8, device="cuda").requires_grad_()
        out = embedding(torch.zeros(ids_shape, dtype=torch.int64, device="cuda"), table, 2.0)
        assert out.shape == (*ids_shape, 8) and not bool(out.any())
        grad, = torch.autograd.grad(out.sum(), table)
        assert grad.shape == table.shape and not bool(grad.any())


def test_another_stream_and_a_graph_of_launches():
    from paper_2605_15695_amd.embedding import _gradient, embedding

    g = _gen(7)
    table = torch.randn(3000, 32, generator=g, device="cuda").requires_grad_()
    ids = torch.randint(0, 3000, (20000,), generator=g, device="cuda")
    dout = torch.randn(20000, 32, generator=g, device="cuda")
    want = embedding(ids, table, 1.5)
    want_grad, = torch.autograd.grad(want, table, dout)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out = embedding(ids, table, 1.5)
        grad, = torch.autograd.grad(out, table, dout)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(grad, want_grad)
    # without autograd's engine: it would have a leaf's stream, which is not captured, wait for the one that is
    table = table.detach()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = embedding(ids, table, 1.5)
        grad = _gradient(ids, dout, table.shape, table.dtype, 1.5)
    for k in range(3):
        table.mul_(1.0 + k)
        dout.mul_(-1.0)
        ids.copy_(ids.flip(0))
        eager, eager_grad = embedding(ids, table, 1.5), _gradient(ids, dout, table.shape, table.dtype, 1.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(grad, eager_grad)


def test_refusals():
    from paper_2605_15695_amd.embedding import embedding

    ids, table = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(4, 5, device="cuda")
    for bad in ((ids.float(), table), (ids.short(), table), (ids, table.double()), (ids, table[0]), (ids, table.cpu()),
                (ids.cpu(), table), (ids, table[:, :0]), ([0, 1], table)):
        with pytest.raises(ValueError):
            embedding(*bad)


def test_module_learns_its_rows():
    from paper_2605_15695_amd.embedding import NodeEmbedding

    torch.manual_seed(0)
    emb = NodeEmbedding(100, 16, scale=4.0, device="cuda")
    assert emb.weight.shape == (100, 16) and abs(float(emb.weight.std()) - 0.25) < 0.03
    ids = torch.arange(0, 100, 2, device="cuda")
    target = torch.randn(50, 16, device="cuda")
    opt = torch.optim.SGD(emb.parameters(), lr=0.02)
    first = None
    for _ in range(40):
        loss = (emb(ids) - target).square().sum()
        first = first or float(loss)
        opt.zero_grad()
        loss.backward()
        assert not bool(emb.weight.grad[1::2].any())
        opt.step()
    assert float(loss) < 1e-3 * first and np.isfinite(first)


# the module of calls on C++ objects, and the Python code that stands in for it
def test_without_the_call_module(monkeypatch):
    from paper_2605_15695_amd import binding
    from paper_2605_15695_amd.embedding import embedding

    g = _gen(12)
    table = torch.randn(300, 40, generator=g, device="cuda").requires_grad_()
    ids = torch.randint(-3, 303, (4, 90), generator=g, device="cuda")
    dout = torch.randn(4, 90, 40, generator=g, device="cuda")
    assert binding.train_module() is not None
    want = embedding(ids, table, 3.0)
    grad, = torch.autograd.grad(want, table, dout)
    monkeypatch.setattr(binding, "_train", None)
    out = embedding(ids, table, 3.0)
    assert torch.equal(out, want) and torch.equal(torch.autograd.grad(out, table, dout)[0], grad)
    monkeypatch.setattr(binding, "_train", False)
    monkeypatch.setattr(binding, "TRAIN_PATH", binding.TRAIN_PATH.with_name("_no_such_module.so"))
    with pytest.warns(RuntimeWarning, match="_no_such_module"):
        assert torch.equal(embedding(ids, table, 3.0), want)


def test_gradients_of_gradients_are_refused():
    from paper_2605_15695_amd.embedding import embedding

    table = torch.randn(10, 4, device="cuda").requires_grad_()
    out = embedding(torch.tensor([1, 2], device="cuda"), table)
    grad, = torch.autograd.grad(out.square().sum(), table, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
