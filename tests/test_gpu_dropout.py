"""Dropout against its definition: which numbers are dropped exactly, the others by arithmetic.

A kept number is a product rounded in fp32, a sum rounded in fp32 and a rounding to its type: off by at most u (2 |f x| + |r|) with
u = 2^-24, and half a step of its type."""
import numpy as np
import pytest

from drop_reference import kept

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}
U = 2.0 ** -24
SEED = 0x9E3779B97F4A7C15


@pytest.fixture(params=["module", "python"])
def path(request, monkeypatch):
    """Both ways to the library: the module of calls on tensors' C++ objects, and the Python code"""
    from paper_2605_15695_amd import binding

    assert binding.train_module() is not None
    if request.param == "python":
        monkeypatch.setattr(binding, "_train", None)
    return request.param


def _normal(seed, *shape, kind="fp32"):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(TYPES[kind][0])


def _factor(shape, p, seed, offset):
    cols = shape[-1]
    k, f = kept(int(np.prod(shape[:-1])), cols, p, seed, offset)
    return torch.from_numpy(k).cuda().view(*shape), f


def _check(out, X, residual, p, seed, offset, kind):
    k, f = _factor(X.shape, p, seed, offset)
    x, r = torch.where(k, X.double() * f, 0.0), torch.zeros_like(X, dtype=torch.float64) if residual is None else residual.double()
    err = U * (2 * x.abs() + r.abs()) + TYPES[kind][1] * (x + r).abs() + 2.0 ** -25
    assert out.shape == X.shape and out.dtype == X.dtype
    assert bool(((out.double() - x - r).abs() <= err).all())
    if residual is None:
        assert bool((out[~k] == 0).all()) and bool((out[k] != 0).eq(X[k] != 0).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 64), (3, 8), (777, 75), (5, 1000), (300, 7), (2000, 16), (70_000, 9), (1, 40_003)])
@pytest.mark.parametrize("residual", [False, True])
def test_rows(path, kind, rows, cols, residual):
    from paper_2605_15695_amd.dropout import dropout

    X, dy = _normal(1, rows, cols, kind=kind), _normal(2, rows, cols, kind=kind)
    R = _normal(3, rows, cols, kind=kind) if residual else None
    for p, seed, offset in ((0.5, 7, 0), (0.1, SEED, (5 << 40) + 3), (0.9, -1, -2)):
        _check(dropout(X, p, seed, offset, R), X, R, p, seed, offset, kind)
        leaves = [t.detach().clone().requires_grad_() for t in (X, R) if t is not None]
        out = dropout(leaves[0], p, seed, offset, leaves[1] if residual else None)
        _check(out.detach(), X, R, p, seed, offset, kind)
        grads = torch.autograd.grad(out, leaves, dy)
        _check(grads[0], dy, None, p, seed, offset, kind)
        assert not residual or torch.equal(grads[1], dy)


# the ends of p: nothing, what rounds to nothing, everything
def test_probabilities(path):
    from paper_2605_15695_amd.dropout import dropout

    X = _normal(4, 500, 64)
    assert torch.equal(dropout(X, 0.0, 1), X) and torch.equal(dropout(X, 2.0 ** -18, 1), X)
    X[3, 5], X[4, 6] = float("nan"), float("inf")
    assert torch.equal(dropout(X, 1.0, 1), torch.zeros_like(X))
    out = dropout(X, 0.5, 1)
    k, _ = _factor(X.shape, 0.5, 1, 0)
    assert bool((out[~k] == 0).all())  # whatever was there
    share = float((dropout(torch.ones(4000, 512, device="cuda"), 0.3, 9) == 0).float().mean())
    assert abs(share - 0.3) < 6 * (0.21 / (4000 * 512)) ** 0.5 + 2.0 ** -17


# rows that lie apart, begin anywhere, are columns of something, or are one number many times
@pytest.mark.parametrize("kind", list(TYPES))
def test_strides(path, kind):
    from paper_2605_15695_amd.dropout import dropout

    big = _normal(5, 100, 90, kind=kind)
    for X in (big[:, 3:78], big[::3, 1:2], big.t()[5:9], big[:, :1].expand(100, 64), big.view(10, 10, 90)[:, 2:7], big.view(10, 10, 90).transpose(0, 1),
              big[7], big[7, ::2], big[:0], big[:, :0]):
        _check(dropout(X, 0.4, 11, 2), X.contiguous(), None, 0.4, 11, 2, kind)
        _check(dropout(X, 0.4, 11, 2, X), X.contiguous(), X.contiguous(), 0.4, 11, 2, kind)
    X = big.clone().requires_grad_()
    dropout(X, 0.4, 11).sum().backward()  # its gradient is one number, expanded
    _check(X.grad, torch.ones_like(big), None, 0.4, 11, 0, kind)
    Z = torch.randn(50, 8, dtype=torch.complex64, device="cuda").conj().imag  # a view with the other sign
    assert Z.is_neg()
    _check(dropout(Z, 0.4, 11), Z.resolve_neg().contiguous(), None, 0.4, 11, 0, "fp32")


def test_seeds_in_device_memory(path):
    from paper_2605_15695_amd.dropout import dropout

    X, dy = _normal(6, 300, 40), _normal(7, 300, 40)
    state = torch.tensor([SEED - (1 << 64), 5], device="cuda")
    X.requires_grad_()
    out = dropout(X, 0.3, state)
    _check(out.detach(), X.detach(), None, 0.3, SEED, 5, "fp32")
    state.add_(1)  # the backward pass uses what the forward pass did
    grad, = torch.autograd.grad(out, X, dy)
    _check(grad, dy, None, 0.3, SEED, 5, "fp32")
    _check(dropout(X, 0.3, state).detach(), X.detach(), None, 0.3, SEED + 1, 6, "fp32")
    both = torch.stack([state, state], 1)[:, 0]  # two numbers that do not lie side by side
    _check(dropout(X, 0.3, both).detach(), X.detach(), None, 0.3, SEED + 1, 6, "fp32")


def test_module_counts_and_resumes(path):
    from paper_2605_15695_amd.dropout import Dropout

    torch.manual_seed(3)
    m, other = Dropout(0.5).cuda(), Dropout(0.5).cuda()
    seed = int(m.counter[0])
    assert int(other.counter[0]) != seed
    X, R = _normal(8, 64, 32), _normal(9, 64, 32)
    for step in range(3):
        _check(m(X), X, None, 0.5, seed, step, "fp32")
    saved = {k: v.clone() for k, v in m.state_dict().items()}
    _check(m(X, R), X, R, 0.5, seed, 3, "fp32")
    other.load_state_dict(saved)
    _check(other(X, R), X, R, 0.5, seed, 3, "fp32")
    m.eval()
    assert m(X) is X and torch.equal(m(X, R), X + R) and int(m.counter[1]) == 4


# a captured forward and backward pass drops others on every replay, beside eager work on the same module
def test_graph_replays(path):
    from paper_2605_15695_amd.dropout import Dropout

    m = Dropout(0.25, seed=21).cuda()
    X, dy = _normal(10, 200, 75).requires_grad_(), _normal(11, 200, 75)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(m(X), X, dy)  # warm, offset 0
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = m(X)
        grad, = torch.autograd.grad(out, X, dy)
    step = 1
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        _check(out.detach(), X.detach(), None, 0.25, 21, step, "fp32")
        _check(grad, dy, None, 0.25, 21, step, "fp32")
        _check(m(X).detach(), X.detach(), None, 0.25, 21, step + 1, "fp32")
        step += 2


def test_streams(path):
    from paper_2605_15695_amd.dropout import dropout

    X = _normal(12, 50_000, 64)
    want = dropout(X, 0.5, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = dropout(X, 0.5, 3)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)


# rows whose numbers lie past 2^31, and more groups than one launch takes: each part of the launches against a call of its own rows
def test_long_arrays(path):
    from paper_2605_15695_amd.dropout import dropout

    for rows, cols in ((1 << 22, 520), ((1 << 31) + 5000, 1)):  # 2.18 thousand million numbers; two launches
        X = torch.ones(rows, cols, device="cuda", dtype=torch.bfloat16)
        out = dropout(X, 0.5, 17, 1)
        for first in (0, rows // 2, rows - 50):
            k, f = kept(50, cols, 0.5, 17, 1, first)  # (rows past 2^31 - 256 are the second launch's)
            assert torch.equal(out[first:first + 50].float().cpu(), torch.from_numpy(k).float() * f)
        del X, out


def test_refusals(path):
    from paper_2605_15695_amd.dropout import Dropout, dropout

    X = _normal(13, 4, 8)
    for bad in (dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(seed=1.0), dict(seed=1 << 64), dict(seed=True), dict(offset=None),
                dict(seed=torch.zeros(2, dtype=torch.int64)), dict(seed=torch.zeros(3, dtype=torch.int64, device="cuda")),
                dict(seed=torch.zeros(2, device="cuda")), dict(residual=X[:2]), dict(residual=X.half()), dict(residual=X.cpu()), dict(X=X.double()),
                dict(X=X.cpu()), dict(X=X[0, 0])):
        with pytest.raises(ValueError):
            dropout(**{**dict(X=X, p=0.5, seed=1), **bad})
    with pytest.raises(ValueError):
        Dropout(1.5)
    x = X.clone().requires_grad_()
    g, = torch.autograd.grad(dropout(x, 0.5, 1).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)
    import torch.autograd.forward_ad as fw

    with fw.dual_level(), pytest.raises((NotImplementedError, RuntimeError)):
        dropout(fw.make_dual(X, X), 0.5, 1)
