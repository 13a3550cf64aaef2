"""Orthogonalised updates and the optimiser on them, against the polynomial in 64 bits.

Errors are 2-norms of differences over the 2-norm of the result.  A rounding of X in the first step can grow by 3.4445 a
step, 485 times in five, where singular values are small: of one rounding to 24 bits that leaves 485 * 2^-24 = 2.9e-5.
Operands of fp32 and fp16 matrices are 22 bits, whose roundings (four times as large) reach such directions only through
products with large ones, so the same bound is asked of them.  bf16 matrices have operands of 11 bits: eight roundings of 2^-12
(two operands in each of three products, less where they cancel) a step's share, and the result's own 2^-8."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BOUND = {torch.float32: 485 * 2.0 ** -24, torch.float16: 485 * 2.0 ** -24 + 2.0 ** -11, torch.bfloat16: 8 * 2.0 ** -12 + 2.0 ** -8}
TYPES = list(BOUND)
QUINTIC = (3.4445, -4.7750, 2.0315)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _polynomial(G, steps=5, co=QUINTIC):
    X = G.double()
    norm = X.norm()
    X = X / norm if float(norm) > 0 else X
    rows = co if isinstance(co[0], tuple) else [co] * steps
    for a, b, c in rows:
        S = X.t().contiguous() @ X if X.shape[0] >= X.shape[1] else X @ X.t().contiguous()
        P = b * S + c * (S @ S)
        X = a * X + (X @ P if X.shape[0] >= X.shape[1] else P @ X)
    return X


def _near(got, want, bound):
    err = float((got.double() - want).norm() / want.norm().clamp_min(1e-300))
    assert err <= bound, err


SHAPES = [(1, 1), (1, 7), (40, 1), (16, 64), (64, 16), (64, 64), (65, 3), (33, 47), (128, 128), (100, 128), (129, 5), (3, 400), (130, 130),
          (100, 300), (1000, 333), (257, 513), (700, 700)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(dtype, shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(sum(shape)), device="cuda").to(dtype)
    out = orthogonalize(G)
    assert out.shape == G.shape and out.dtype == dtype
    _near(out, _polynomial(G), BOUND[dtype])
    assert torch.equal(out, orthogonalize(G))


# enough tiles of 128 for every compute unit
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(2048, 1500), (1537, 2300)])
def test_large_matrices(dtype, shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(1), device="cuda").to(dtype)
    _near(orthogonalize(G), _polynomial(G), BOUND[dtype])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(3, 20, 30), (30, 64, 40), (5, 300, 200), (26, 140, 20), (2, 129, 129)])
def test_stacks(dtype, shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(7), device="cuda") * torch.logspace(-3, 3, shape[0], device="cuda").view(-1, 1, 1)
    G = G.to(dtype)
    G[1] = 0
    out = orthogonalize(G)
    assert not bool(out[1].any())
    for k in range(shape[0]):
        if k != 1:
            _near(out[k], _polynomial(G[k]), BOUND[dtype])
            assert k > 2 or torch.equal(out[k], orthogonalize(G[k])) or shape[1] > 128


@pytest.mark.parametrize("shape", [(40, 60), (200, 150)])
def test_any_scale_and_its_ends(shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(2), device="cuda")
    want = _polynomial(G)
    for scale in (2.0 ** 124, 2.0 ** -100):  # squares beyond and below fp32
        _near(orthogonalize(G * scale), want, BOUND[torch.float32])
    small = G * 2.0 ** -140  # numbers without a leading bit
    _near(orthogonalize(small), _polynomial(small), BOUND[torch.float32])
    for bad in (float("nan"), float("inf")):
        G[3, 4] = bad
        assert not bool(torch.isfinite(orthogonalize(G)).any())


@pytest.mark.parametrize("shape", [(48, 100), (150, 260)])
def test_few_directions(shape):
    from paper_2605_15695_amd.muon import orthogonalize

    g = _gen(3)
    for rank in (1, 3):
        G = torch.randn(shape[0], rank, generator=g, device="cuda") @ torch.randn(rank, shape[1], generator=g, device="cuda")
        # the rounding of G itself is a matrix of full rank, which both sides have; theirs adds sqrt(side) directions of it
        _near(orthogonalize(G), _polynomial(G), BOUND[torch.float32] * math.sqrt(min(shape)))
        H = G.to(torch.bfloat16)
        _near(orthogonalize(H), _polynomial(H), BOUND[torch.bfloat16] * math.sqrt(min(shape)))


@pytest.mark.parametrize("shape", [(30, 50), (300, 170)])
def test_other_polynomials(shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(4), device="cuda")
    cubic = (1.5, -0.5, 0.0)
    for steps, co in ((1, QUINTIC), (3, [QUINTIC, (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]), (16, cubic), (2, (0.0, 0.0, 0.0)), (2, (9.0, -3.0, 0.5))):
        want = _polynomial(G, steps, tuple(map(tuple, co)) if isinstance(co, list) else co)
        _near(orthogonalize(G, steps, co), want, BOUND[torch.float32] * 4)
    # a cubic that converges from a spectrum away from 0 makes the rows orthonormal
    Q, _ = torch.linalg.qr(torch.randn(max(shape), min(shape), generator=_gen(5), device="cuda"))
    H = (Q * torch.linspace(0.5, 1.5, min(shape), device="cuda")).contiguous()
    O = orthogonalize(H, 16, cubic).double()
    eye = torch.eye(min(shape), device="cuda", dtype=torch.float64)
    assert float((O.t().contiguous() @ O - eye).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", TYPES)
def test_strides(dtype):
    from paper_2605_15695_amd.muon import orthogonalize

    big = torch.randn(4, 300, 410, generator=_gen(6), device="cuda").to(dtype)
    for G in (big[0, 3:103, 7:90], big[1].t(), big[:, ::3, 1:200], big[2, :, ::5], big[3, :1].expand(20, 410)):
        want = torch.stack([_polynomial(x) for x in G]) if G.dim() == 3 else _polynomial(G)
        _near(orthogonalize(G), want, BOUND[dtype] * (1 if G.stride(0) else math.sqrt(20)))


def test_empty_and_refusals():
    import paper_2605_15695_amd as pc
    from paper_2605_15695_amd.muon import Muon, orthogonalize

    for shape in ((0, 5), (5, 0), (0, 3, 4), (2, 0, 4)):
        assert orthogonalize(torch.empty(shape, device="cuda")).shape == shape
    G = torch.ones(4, 4, device="cuda")
    for args in ((G.double(),), (G[0],), (G.cpu(),), (G, 0), (G, 17), (G, 2.0), (G, 2, (1.0, 2.0)), (G, 2, [QUINTIC] * 3)):
        with pytest.raises(ValueError):
            orthogonalize(*args)
    for co in ((1e9, 0.0, 0.0), (float("nan"), 0.0, 0.0), (30.0, 40.0, 50.0)):
        with pytest.raises(pc.PcsrError):
            orthogonalize(G, 5, co)
    p = torch.nn.Parameter(G.clone())
    for kw in (dict(lr=-1.0), dict(momentum=1.0), dict(weight_decay=-0.1), dict(steps=0), dict(coefficients=(1.0,))):
        with pytest.raises(ValueError):
            Muon([p], **kw)
    for bad in (torch.nn.Parameter(torch.zeros(3, device="cuda")), torch.nn.Parameter(torch.zeros(2, 2, device="cuda", dtype=torch.float64))):
        with pytest.raises(ValueError):
            Muon([bad])
    host = torch.nn.Parameter(torch.ones(2, 2))
    host.grad = torch.ones(2, 2)
    with pytest.raises(ValueError):
        Muon([host]).step()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nesterov,momentum,decay", [(True, 0.95, 0.0), (False, 0.9, 0.1), (True, 0.0, 0.01)])
def test_optimiser_against_64_bits(dtype, nesterov, momentum, decay):
    from paper_2605_15695_amd.muon import Muon

    g = _gen(8)
    shapes = [(64, 16)] + [(64, 64)] * 27 + [(16, 64), (128, 100), (300, 140), (140, 300), (300, 140), (200, 1)]
    params = [torch.nn.Parameter(torch.randn(*s, generator=g, device="cuda").to(dtype)) for s in shapes]
    params.append(torch.nn.Parameter(torch.randn(90, 70, generator=g, device="cuda").to(dtype)[:, 5:41]))
    params.append(torch.nn.Parameter(torch.randn(20, 30, generator=g, device="cuda").to(dtype).t()))
    idle = torch.nn.Parameter(torch.ones(5, 5, device="cuda", dtype=dtype))
    lr = 0.1
    opt = Muon(params + [idle], lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=decay)
    bufs = [torch.zeros(p.shape, device="cuda", dtype=torch.float64) for p in params]
    for _ in range(3):
        was = [p.detach().double() for p in params]
        for p in params:
            p.grad = torch.randn(*p.shape, generator=g, device="cuda").to(dtype)
        opt.step()
        for k, (p, w) in enumerate(zip(params, was)):
            bufs[k] = momentum * bufs[k] + p.grad.double()
            O = _polynomial(p.grad.double() + momentum * bufs[k] if nesterov else bufs[k])
            gain = max(1.0, p.shape[0] / p.shape[1]) ** 0.5
            want = w * (1.0 - lr * decay) - lr * gain * O
            # the update's error, and the weight's own rounding
            u = {torch.float32: 2.0 ** -23, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
            off = float((p.detach().double() - want).norm())
            assert off <= BOUND[dtype] * lr * gain * float(O.norm()) + u * float(want.norm()), (k, off)
            state = opt.state[p]["momentum"]
            assert state.dtype == torch.float32
            _near(state, bufs[k], 4 * 2.0 ** -24)
    assert bool((idle == 1).all())


def test_optimiser_state_goes_through_a_checkpoint():
    from paper_2605_15695_amd.muon import Muon

    g = _gen(9)
    start, grads = torch.randn(70, 150, generator=g, device="cuda"), [torch.randn(70, 150, generator=g, device="cuda") for _ in range(4)]

    def steps(p, opt, gs):
        for x in gs:
            p.grad = x
            opt.step()

    p = torch.nn.Parameter(start.clone())
    opt = Muon([p])
    steps(p, opt, grads[:2])
    q = torch.nn.Parameter(p.detach().clone())
    other = Muon([q], lr=5.0)
    other.load_state_dict(opt.state_dict())
    steps(p, opt, grads[2:])
    steps(q, other, grads[2:])
    assert torch.equal(p, q)
    first = torch.nn.Parameter(torch.randn(20, 20, generator=g, device="cuda").to(torch.bfloat16))  # load_state_dict casts state to bf16
    opt = Muon([first])
    steps(first, opt, [torch.ones(20, 20, device="cuda", dtype=torch.bfloat16)])
    opt.load_state_dict(opt.state_dict())
    steps(first, opt, [torch.ones(20, 20, device="cuda", dtype=torch.bfloat16)])
    assert opt.state[first]["momentum"].dtype == torch.float32


def test_another_stream_and_a_graph_of_launches():
    from paper_2605_15695_amd.muon import orthogonalize

    Gs = [torch.randn(60, 90, generator=_gen(10), device="cuda"), torch.randn(3, 200, 300, generator=_gen(11), device="cuda")]
    want = [orthogonalize(G) for G in Gs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [orthogonalize(G) for G in Gs]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [orthogonalize(G) for G in Gs]
    for _ in range(3):
        for G in Gs:
            G.copy_(G.flip(-1)).add_(0.01)
        want = [orthogonalize(G) for G in Gs]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_model_learns():
    from paper_2605_15695_amd.muon import Muon

    torch.manual_seed(0)
    model = torch.nn.Sequential(torch.nn.Linear(16, 64), torch.nn.ReLU(), torch.nn.Linear(64, 16)).cuda()
    X = torch.randn(500, 16, device="cuda")
    Y = torch.tanh(X @ torch.randn(16, 16, device="cuda"))
    opts = [Muon([p for p in model.parameters() if p.dim() == 2], lr=0.02), torch.optim.Adam([p for p in model.parameters() if p.dim() == 1], 1e-3)]
    losses = []
    for _ in range(60):
        loss = torch.nn.functional.mse_loss(model(X), Y)
        for o in opts:
            o.zero_grad()
        loss.backward()
        for o in opts:
            o.step()
        losses.append(float(loss.detach()))
    assert losses[-1] < 0.3 * losses[0]


# the module of calls on C++ objects, and the Python code that stands in for it
def test_without_the_call_module(monkeypatch):
    from paper_2605_15695_amd import binding
    from paper_2605_15695_amd.muon import Muon, orthogonalize

    assert binding.train_module() is not None
    g = _gen(13)
    G = torch.randn(3, 50, 70, generator=g, device="cuda")
    start = [torch.randn(s, generator=g, device="cuda") for s in ((20, 30), (200, 140))]
    grads = [torch.randn(p.shape, generator=g, device="cuda") for p in start]

    def run():
        params = [torch.nn.Parameter(p.clone()) for p in start]
        opt = Muon(params, lr=0.1)
        for p, x in zip(params, grads):
            p.grad = x
        versions = [p._version for p in params]
        opt.step()
        opt.step()
        assert all(p._version > v for p, v in zip(params, versions))
        return [p.detach() for p in params] + [orthogonalize(G), orthogonalize(G[1])]

    want = run()
    monkeypatch.setattr(binding, "_train", None)
    assert all(torch.equal(a, b) for a, b in zip(run(), want))
