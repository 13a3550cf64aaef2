"""Group norm with an activation against plain torch in 64 bits.

With u = 2^-24: mean and rstd are rounded once from sums in 64 bits, xhat is a difference and a product, z a
product and a sum, so z is off by at most u * (6 |xhat w| + 3 |mean| rstd |w| + 2 |b|); the activations' slopes are at most
1.13, and their own exponentials and divisions are good to u * 8 (1 + |z|) |z|.  Gradients: slopes are off by u * 16 (1 + |z|)
and, through z, by the error above (second derivatives are at most 0.8); sums of up to a few thousand products in chains of at
most a few hundred are off by 64 u of the sum of their magnitudes where roundings add up as random ones do, four times what
chains of 256 give.  Results are then rounded to their type."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}
U = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _act(z, name):
    return {"none": lambda v: v * 1.0, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
            "gelu": lambda v: 0.5 * v * torch.erfc(-v / 2.0 ** 0.5)}[name](z)


class Plain:
    """In 64 bits: y, dx, dw, db, and what their roundings scale with"""

    def __init__(self, X, groups, weight, bias, lengths, eps, act, dy):
        C = X.shape[-1]
        x, g = X.detach().double().reshape(-1, C), dy.detach().double().reshape(-1, C)
        w = torch.ones(C, dtype=torch.float64, device="cuda") if weight is None else weight.detach().double()
        b = torch.zeros(C, dtype=torch.float64, device="cuda") if bias is None else bias.detach().double()
        outs = {k: torch.zeros_like(x) for k in ("y", "dx", "z_err", "dx_size", "xhat", "dz")}
        at = 0
        for n in lengths:
            s, at = slice(at, at + n), at + n
            if n == 0:
                continue
            v = x[s].view(n, groups, -1)
            mean, var = v.mean((0, 2), keepdim=True), v.var((0, 2), unbiased=False, keepdim=True)
            rstd = 1.0 / torch.sqrt(var + eps)
            xhat = (v - mean) * rstd
            wv, bv = w.view(1, groups, -1), b.view(1, groups, -1)
            z = (xhat * wv + bv).requires_grad_()
            y = _act(z, act)
            slope, = torch.autograd.grad(y.sum(), z)
            z, y = z.detach(), y.detach()
            gv = g[s].view(n, groups, -1)
            dz = gv * slope
            d = dz * wv
            m = v.shape[0] * v.shape[2]
            dx = rstd * (d - d.sum((0, 2), keepdim=True) / m - xhat * (d * xhat).sum((0, 2), keepdim=True) / m)
            z_err = U * (6 * (xhat * wv).abs() + 3 * mean.abs() * rstd * wv.abs() + 2 * bv.abs())
            own = U * 8 * (1 + z.abs()) * z.abs()
            slope_err = (gv * wv).abs() * (16 * U * (1 + z.abs()) + 0.8 * z_err)
            x_err = (3 * mean.abs() * rstd + 4 * xhat.abs()) * U
            size = rstd * (slope_err + slope_err.mean((0, 2), keepdim=True) + xhat.abs() * (slope_err * xhat.abs()).mean((0, 2), keepdim=True)
                           + 64 * U * (d.abs() + d.abs().mean((0, 2), keepdim=True) + xhat.abs() * (d * xhat).abs().mean((0, 2), keepdim=True))
                           + x_err * (d * xhat).abs().mean((0, 2), keepdim=True) + xhat.abs() * (d.abs() * x_err).mean((0, 2), keepdim=True))
            for k, t in (("y", y), ("dx", dx), ("z_err", 1.13 * z_err + own), ("dx_size", size), ("xhat", xhat), ("dz", dz)):
                outs[k][s] = t.reshape(n, C)
            outs.setdefault("dw_err", torch.zeros(C, dtype=torch.float64, device="cuda")).add_(
                ((slope_err / wv.abs().clamp_min(1e-30) * xhat.abs() + dz.abs() * x_err)).sum(0).reshape(C))
            outs.setdefault("db_err", torch.zeros(C, dtype=torch.float64, device="cuda")).add_((slope_err / wv.abs().clamp_min(1e-30)).sum(0).reshape(C))
        self.__dict__.update(outs)
        self.dw, self.db = (self.dz * self.xhat).sum(0), self.dz.sum(0)
        self.dw_err = self.dw_err + 64 * U * (self.dz * self.xhat).abs().sum(0)
        self.db_err = self.db_err + 64 * U * self.dz.abs().sum(0)


def _near(got, want, err, u):
    far = (got.detach().double().reshape(want.shape) - want).abs() - (err + u * (want.abs() + err) + 2.0 ** -25)
    assert bool((far <= 0).all()), float(far.max())


def _check(X, groups, weight, bias, lengths, offsets, act, kind, eps=1e-5, dy=None):
    from paper_2605_15695_amd.norm import group_norm

    u = TYPES[kind][1]
    g = _gen(11)
    if dy is None:
        dy = torch.randn(X.shape, generator=g, device="cuda").to(X.dtype)
    ref = Plain(X, groups, weight, bias, lengths, eps, act, dy)
    leaves = [None if t is None else t.detach().requires_grad_() for t in (X, weight, bias)]
    y = group_norm(leaves[0], groups, leaves[1], leaves[2], offsets, eps, act)
    assert y.shape == X.shape and y.dtype == X.dtype
    _near(y, ref.y, ref.z_err, u)
    with torch.no_grad():
        assert torch.equal(group_norm(leaves[0], groups, leaves[1], leaves[2], offsets, eps, act), y)
    want = [t for t in leaves if t is not None]
    grads = list(torch.autograd.grad(y, want, dy, retain_graph=True))
    assert all(torch.equal(a, b) for a, b in zip(grads, torch.autograd.grad(y, want, dy, retain_graph=True)))
    if len(want) > 1:  # one at a time
        for t, whole in zip(want, grads):
            assert torch.equal(torch.autograd.grad(y, t, dy, retain_graph=True)[0], whole)
    _near(grads.pop(0), ref.dx, ref.dx_size, u)
    if weight is not None:
        _near(grads.pop(0), ref.dw, ref.dw_err, U if weight.dtype == torch.float32 else u)
    if bias is not None:
        _near(grads.pop(0), ref.db, ref.db_err, U if bias.dtype == torch.float32 else u)


def _offsets(lengths, wide=True):
    return torch.tensor([0] + list(lengths), device="cuda").cumsum(0).to(torch.int64 if wide else torch.int32)


def _inputs(seed, n, C, kind, shift=1.0):
    g = _gen(seed)
    X = (torch.randn(n, C, generator=g, device="cuda") + shift * torch.randn(C, generator=g, device="cuda")).to(TYPES[kind][0])
    return X, 1.0 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")


# one graph: in registers, read again by its workgroup, cut into chunks
@pytest.mark.parametrize("kind,act", [("fp32", "relu"), ("fp32", "gelu"), ("bf16", "silu"), ("fp16", "none"), ("fp16", "gelu")])
@pytest.mark.parametrize("C,groups", [(1, 1), (6, 2), (64, 8), (64, 1), (75, 5), (320, 32), (2048, 1), (33, 33), (1030, 2)])
@pytest.mark.parametrize("n", [1, 5, 24, 300, 2500])
def test_one_graph(kind, act, C, groups, n):
    if n * C > 700_000:
        n = 700_000 // C
    X, w, b = _inputs(n + C, n, C, kind)
    _check(X, groups, w, b, [n], None, act, kind)


@pytest.mark.parametrize("kind,act", [("fp32", "silu"), ("bf16", "relu"), ("fp16", "gelu"), ("fp32", "none")])
@pytest.mark.parametrize("C,groups", [(64, 8), (20, 4), (7, 7), (256, 2)])
@pytest.mark.parametrize("lengths", [[1], [0, 3, 0], [1] * 9, [0, 0, 17, 1, 0, 63, 64, 65, 2], [5, 4000, 3, 0, 1, 2500, 7],
                                     [24] * 700 + [0] * 5 + [9000]])
def test_ragged_graphs(kind, act, C, groups, lengths):
    wide = (C + len(lengths)) % 2 == 0
    if sum(lengths) * C > 1_200_000:
        lengths = lengths[-60:]
    X, w, b = _inputs(sum(lengths) + C, sum(lengths), C, kind)
    _check(X, groups, w, b, lengths, _offsets(lengths, wide), act, kind)


@pytest.mark.parametrize("shape,groups", [((3, 40, 16), 4), ((2, 9, 11, 24), 3), ((5, 1, 12), 1), ((2, 3000, 48), 6), ((1, 7, 8), 2)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_stacks(shape, groups, kind):
    X, w, b = _inputs(3, int(torch.Size(shape[:-1]).numel()), shape[-1], kind)
    n = X.shape[0] // shape[0]
    _check(X.view(shape), groups, w, b, [n] * shape[0], None, "silu", kind)


def test_many_small_graphs_share_workgroups():
    lengths = [2 + (k * 7) % 5 for k in range(6000)]
    X, w, b = _inputs(1, sum(lengths), 16, "fp32")
    _check(X, 2, w, b, lengths, _offsets(lengths), "silu", "fp32")


@pytest.mark.parametrize("w_type,b_type", [(None, None), ("fp32", None), (None, "fp32"), ("bf16", "bf16")])
def test_weights_of_other_types_or_none(w_type, b_type):
    X, w, b = _inputs(4, 90, 24, "bf16")
    w = None if w_type is None else w.to(TYPES[w_type][0])
    b = None if b_type is None else b.to(TYPES[b_type][0])
    _check(X, 3, w, b, [50, 0, 40], _offsets([50, 0, 40]), "gelu", "bf16")


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_and_alignment(kind):
    X, w, b = _inputs(9, 130, 201, kind)
    for x in (X[:, 1:49], X[:, ::2][:, :48], X.t()[:128, :48], X[::2, 3:51], X[:1, :48].expand(60, 48)):
        n = x.shape[0]
        wide = torch.randn(n, 97, generator=_gen(1), device="cuda").to(x.dtype)
        _check(x, 4, w[:96:2], b[1:49], [20, n - 20], _offsets([20, n - 20]), "silu", kind, dy=wide[:, 49:])
    _check(X[:, :48], 4, w[:48], b[:48], [130], None, "gelu", kind, dy=torch.ones(1, 1, device="cuda", dtype=X.dtype).expand(130, 48))


# numbers far from 0: the variance is 1e-6 of the mean's square
def test_variance_of_numbers_far_from_zero():
    for n in (40, 6000):
        X, w, b = _inputs(8, n, 32, "fp32", shift=0.0)
        _check(X + 1000.0, 4, w, b, [n], None, "none", "fp32")


def test_a_group_of_one_number_has_no_gradient():
    X, w, b = _inputs(2, 5, 8, "fp32")
    from paper_2605_15695_amd.norm import group_norm

    x = X.clone().requires_grad_()
    y = group_norm(x, 8, w, b, _offsets([1] * 5))
    assert torch.equal(y, b.expand(5, 8))
    dx, = torch.autograd.grad(y, x, torch.randn(5, 8, device="cuda"))
    assert not bool(dx.any())


@pytest.mark.parametrize("lengths", [[6, 5, 7], [3000, 5, 2800]])
def test_infinities_and_nan_stay_in_their_groups(lengths):
    from paper_2605_15695_amd.norm import group_norm

    n = sum(lengths)
    X, w, b = _inputs(6, n, 32, "fp32")
    off, dy = _offsets(lengths), torch.randn(n, 32, generator=_gen(3), device="cuda")
    x = X.clone().requires_grad_()
    y = group_norm(x, 4, w, b, off, activation="silu")
    dx, = torch.autograd.grad(y, x, dy)
    bad = X.clone()
    bad[2, 3], bad[lengths[0] + 1, 30] = float("inf"), float("nan")
    x = bad.requires_grad_()
    z = group_norm(x, 4, w, b, off, activation="silu")
    dz, = torch.autograd.grad(z, x, dy)
    hit = torch.zeros(n, 32, dtype=torch.bool, device="cuda")
    hit[:lengths[0], :8] = True
    hit[lengths[0]:lengths[0] + lengths[1], 24:] = True
    assert torch.equal(y[~hit], z[~hit]) and torch.equal(dx[~hit], dz[~hit])
    assert not bool(torch.isfinite(z[hit]).any())


def test_gradients_are_differences_of_the_function():
    from paper_2605_15695_amd.norm import group_norm

    lengths = [7, 0, 4]
    X, w, b = _inputs(21, 11, 12, "fp32")
    dy = torch.randn(11, 12, generator=_gen(5), device="cuda")
    leaves = [t.clone().requires_grad_() for t in (X, w, b)]
    grads = torch.autograd.grad(group_norm(leaves[0], 3, leaves[1], leaves[2], _offsets(lengths), activation="gelu"), leaves, dy)

    def value(ts):
        return float((group_norm(ts[0], 3, ts[1], ts[2], _offsets(lengths), activation="gelu").double() * dy.double()).sum())

    h = 2.0 ** -7  # third derivatives below 100: h^2 / 6 * 100 = 1e-3; roundings 2^-24 * 132 / h = 1e-3
    for t, grad in enumerate(grads):
        for k in (0, 5, grad.numel() - 1):
            up, down = ([v.clone() for v in (X, w, b)] for _ in range(2))
            up[t].view(-1)[k] += h
            down[t].view(-1)[k] -= h
            assert abs((value(up) - value(down)) / (2 * h) - float(grad.reshape(-1)[k])) < 5e-3


def test_empty_inputs():
    from paper_2605_15695_amd.norm import group_norm

    w, b = torch.ones(8, device="cuda").requires_grad_(), torch.zeros(8, device="cuda").requires_grad_()
    for shape, off in (((0, 8), None), ((0, 8), torch.zeros(4, dtype=torch.int64, device="cuda")), ((0, 8), torch.zeros(1, dtype=torch.int64)),
                       ((3, 0, 8), None), ((0, 5, 8), None)):
        x = torch.empty(shape, device="cuda").requires_grad_()
        y = group_norm(x, 2, w, b, off)
        assert y.shape == shape
        dx, dw, db = torch.autograd.grad(y.sum(), (x, w, b))
        assert dx.shape == shape and not bool(dw.any()) and not bool(db.any())


def test_another_stream_and_a_graph_of_launches():
    from paper_2605_15695_amd.norm import _backward, _forward, group_norm

    lengths = [24] * 100 + [4000]
    X, w, b = _inputs(13, sum(lengths), 32, "fp32")
    off, dy = _offsets(lengths), torch.randn(sum(lengths), 32, generator=_gen(2), device="cuda")
    leaves = [t.requires_grad_() for t in (X, w, b)]

    def step():
        y = group_norm(X, 4, w, b, off, activation="relu")
        return [y, *torch.autograd.grad(y, leaves, dy)]

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    # without autograd's engine: it would have a leaf's stream, which is not captured, wait for the one that is
    X, w, b = (t.detach() for t in leaves)

    def plain_step():
        y, stats, graphs = _forward(X, w, b, 4, off, 1e-5, 1)
        return [y, *_backward(X, w, b, off, stats, dy, 4, 1e-5, 1, graphs, (True, True, True))]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = plain_step()
    for k in range(3):
        X.mul_(1.0 + k).add_(0.1)
        dy.mul_(-1.0)
        want = plain_step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_offsets_that_do_not_ascend_stay_inside_the_arrays():
    from paper_2605_15695_amd.norm import group_norm

    X, w, b = _inputs(1, 100, 16, "fp32")
    off = torch.tensor([5, 90, 30, -7, 1000, 60], device="cuda")
    y = group_norm(X, 2, w, b, off)
    torch.cuda.synchronize()
    assert y.shape == X.shape


def test_refusals():
    import paper_2605_15695_amd as pc
    from paper_2605_15695_amd.norm import GroupNorm, group_norm

    X, w = torch.zeros(10, 12, device="cuda"), torch.zeros(12, device="cuda")
    off = torch.tensor([0, 4, 10], device="cuda")
    for args, more in (((X, 5), {}), ((X, 0), {}), ((X.double(), 2), {}), ((X.cpu(), 2), {}), ((X[0], 2), {}), ((X, 2, w[:6]), {}),
                       ((X, 2, w.half()), {}), ((X, 2, w, w.cpu()), {}), ((X, 2), dict(activation="tanh")), ((X, 2), dict(eps=-1.0)),
                       ((X, 2), dict(eps=float("nan"))), ((X, 2), dict(offsets=off.float())), ((X, 2), dict(offsets=off.cpu() + 1)),
                       ((X, 2), dict(offsets=torch.tensor([0, 7, 3, 10]))), ((X, 2), dict(offsets=off[:1])),
                       ((X.view(2, 5, 12), 2), dict(offsets=off)), ((X, 2.0), {})):
        with pytest.raises(ValueError):
            group_norm(*args, **more)
    with pytest.raises(pc.PcsrError):
        group_norm(torch.zeros(3, 2049, device="cuda"), 1)
    for bad in ((5, 12, 1e-5, "relu"), (2, 12, 1e-5, "tanh")):
        with pytest.raises(ValueError):
            GroupNorm(*bad)


def test_module_between_layers():
    from paper_2605_15695_amd.norm import GroupNorm, group_norm

    norm = GroupNorm(4, 32, activation="relu").cuda()
    X, _, _ = _inputs(3, 50, 32, "fp32")
    off = _offsets([20, 30])
    assert torch.equal(norm(X, off), group_norm(X, 4, norm.weight, norm.bias, off, activation="relu"))
    norm(X).square().sum().backward()
    assert norm.weight.grad.shape == (32,) and norm.bias.grad.shape == (32,)


# the module of calls on C++ objects, and the Python code that stands in for it
def test_without_the_call_module(monkeypatch):
    from paper_2605_15695_amd import binding
    from paper_2605_15695_amd.norm import group_norm

    assert binding.train_module() is not None
    for lengths, shape in (([40, 0, 60], None), ([50, 50], (2, 50, 24))):
        X, w, b = _inputs(14, 100, 24, "bf16")
        X = X if shape is None else X.view(shape)
        off = _offsets(lengths) if shape is None else None
        leaves = [t.requires_grad_() for t in (X, w, b)]

        def step():
            y = group_norm(X, 3, w, b, off, activation="gelu")
            return [y, *torch.autograd.grad(y, leaves, torch.ones_like(y))]

        want = step()
        with monkeypatch.context() as m:
            m.setattr(binding, "_train", None)
            assert all(torch.equal(a, c) for a, c in zip(step(), want))


def test_gradients_of_gradients_are_refused():
    from paper_2605_15695_amd.norm import group_norm

    X = torch.randn(10, 4, device="cuda").requires_grad_()
    grad, = torch.autograd.grad(group_norm(X, 2).square().sum(), X, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
