"""Calls of the operators around the graph layers at the ends of what they take: tables of a few bytes, infinite scales, tangents,
refusals by either call path, views, numbers of matrices and groups beyond one launch."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.fixture(params=["module", "python"])
def path(request, monkeypatch):
    """Both ways to the library: the module of calls on tensors' C++ objects, and the Python code"""
    from paper_2605_15695_amd import binding

    assert binding.train_module() is not None
    if request.param == "python":
        monkeypatch.setattr(binding, "_train", None)
    return request.param


# the products of the same numbers in fp32, rounded once: the same tiles, the same order
@pytest.mark.parametrize("shape", [(256, 300), (700, 520), (4, 600, 520), (14, 1000, 900), (1100, 1930), (40, 30), (300, 200)])
def test_bf16_matrices_have_the_products_of_fp32_ones(path, shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(sum(shape)), device="cuda").to(torch.bfloat16)
    assert torch.equal(orthogonalize(G), orthogonalize(G.float()).to(torch.bfloat16))


# exact matrices of few directions in bf16 (whole numbers): neither roundings that do not average out nor directions that grow out of them
@pytest.mark.parametrize("shape", [(300, 400), (520, 700), (5, 800, 780)])
@pytest.mark.parametrize("rank", [1, 3])
def test_few_directions_of_large_bf16_matrices(path, shape, rank):
    from paper_2605_15695_amd.muon import orthogonalize
    from test_gpu_muon import BOUND, _near, _polynomial

    g = _gen(rank)
    left, right = (torch.randint(0, 2, s, generator=g, device="cuda").float() * 2 - 1 for s in ((*shape[:-1], rank), (*shape[:-2], rank, shape[-1])))
    G = (left @ right).to(torch.bfloat16)
    out = orthogonalize(G)
    for x, o in zip(G if G.dim() == 3 else G[None], out if G.dim() == 3 else out[None]):
        _near(o, _polynomial(x), BOUND[torch.bfloat16])


# tables of 1 to 17 bytes, more ids than one launch looks through: rows without an id are zeros
@pytest.mark.parametrize("kind,rows,d", [("fp32", 3, 1), ("fp32", 1, 3), ("fp32", 1, 1), ("bf16", 7, 1), ("fp16", 2, 3), ("bf16", 8, 1), ("fp16", 9, 1)])
@pytest.mark.parametrize("n", [4097, 5000, 16384, 20000, 70000])
@pytest.mark.parametrize("wide", [False, True])
def test_gradients_of_tables_of_a_few_bytes(kind, rows, d, n, wide):
    from paper_2605_15695_amd import binding as pc

    lib, number = pc._lib(), list(TYPES).index(kind)
    dout = torch.ones(n, d, device="cuda", dtype=TYPES[kind])
    ws = torch.empty(lib.pcsr_embed_workspace(n, rows, d), dtype=torch.uint8, device="cuda")
    for which in (-1, rows, rows - 1):  # no row has an id; the last one has one
        ids = torch.full((n,), -1, device="cuda", dtype=torch.int64 if wide else torch.int32)
        ids[n // 2] = which
        grad = torch.full((rows, d), float("nan"), device="cuda", dtype=TYPES[kind])
        rc = lib.pcsr_embed_backward(n, rows, d, number, ids.data_ptr(), int(wide), dout.data_ptr(), d, 1.0, grad.data_ptr(), ws.data_ptr(),
                                     torch.cuda.current_stream().cuda_stream)
        want = torch.zeros(rows, d, device="cuda", dtype=TYPES[kind])
        if 0 <= which < rows:
            want[which] = 1.0
        assert rc == pc.PCSR_OK and torch.equal(grad, want)


# more groups than a launch has workgroups for in its second dimension (65,535 of 8), over long graphs
@pytest.mark.parametrize("lengths", [[12], [13, 0, 1, 15]])
def test_norms_of_half_a_million_groups(path, lengths):
    from paper_2605_15695_amd.norm import group_norm

    n, C = sum(lengths), 524_320
    g = _gen(n)
    X, dy = torch.randn(n, C, generator=g, device="cuda"), torch.randn(n, C, generator=g, device="cuda")
    off = torch.tensor([0] + lengths, device="cuda").cumsum(0) if len(lengths) > 1 else None
    x, w, b = X.clone().requires_grad_(), (torch.ones(C, device="cuda") * 1.5).requires_grad_(), torch.zeros(C, device="cuda").requires_grad_()
    y = group_norm(x, C, w, b, off)
    dx, dw, db = torch.autograd.grad(y, (x, w, b), dy)
    dw64 = torch.zeros(C, dtype=torch.float64, device="cuda")
    at = 0
    for k in lengths:
        if k == 0:
            continue
        v, gv = X[at:at + k].double(), dy[at:at + k].double()
        rstd = (v.var(0, unbiased=False) + 1e-5).rsqrt()
        xhat, d = (v - v.mean(0)) * rstd, gv * 1.5
        # xhat is 4 at most, mean and products are rounded a dozen times; rstd is 316 at most (a graph of one row, whose numbers are 0)
        want = rstd * (d - d.mean(0) - xhat * (d * xhat).mean(0))
        assert float((y.detach()[at:at + k] - 1.5 * xhat).abs().max()) < 64 * U * (1 + float((v.abs().amax(0) * rstd).max()))
        if k > 1:
            err = (dx[at:at + k] - want).abs() / (rstd * (1 + v.abs().amax(0) * rstd) * 8)
            assert float(err.max()) < 64 * U
        dw64 += (gv * xhat).sum(0)
        at += k
    assert torch.allclose(db.double(), dy.double().sum(0), atol=64 * U * 8, rtol=0)
    assert float(((dw.double() - dw64).abs()).max()) < 1e-2


# as many workgroups to add up chunks of long graphs as a launch has threads for (2^24 of 256)
def test_norms_of_many_groups_in_many_chunks(path):
    from paper_2605_15695_amd.norm import group_norm

    n, C, cut = 4096, 131_300, 3000
    g = _gen(9)
    X, dy = torch.randn(n, C, generator=g, device="cuda"), torch.randn(n, C, generator=g, device="cuda")
    off = torch.tensor([0, cut, n], device="cuda")
    x = X.requires_grad_()
    w, b = torch.ones(C, device="cuda").requires_grad_(), torch.zeros(C, device="cuda").requires_grad_()
    y = group_norm(x, C, w, b, off)
    dx, dw, db = torch.autograd.grad(y, (x, w, b), dy)
    for some in (slice(0, 40), slice(65_000, 65_040), slice(C - 40, C)):  # groups are single channels
        dw64 = torch.zeros(40, dtype=torch.float64, device="cuda")
        for rows in (slice(0, cut), slice(cut, n)):
            v, d = X[rows, some].detach().double(), dy[rows, some].double()
            rstd = (v.var(0, unbiased=False) + 1e-5).rsqrt()
            xhat = (v - v.mean(0)) * rstd
            want = rstd * (d - d.mean(0) - xhat * (d * xhat).mean(0))
            # numbers of 5 at most, sums of thousands: roundings of 64 u of sizes of up to 25
            assert float((y.detach()[rows, some] - xhat).abs().max()) < 64 * U * 25
            assert float((dx[rows, some] - want).abs().max()) < 64 * U * 25
            dw64 += (d * xhat).sum(0)
        assert float((dw[some] - dw64).abs().max()) < 64 * U * n
        assert float((db[some] - dy[:, some].double().sum(0)).abs().max()) < 64 * U * n


# 2^30 ids, 16 lanes to a row by its width: as many threads as no launch has
def test_a_lookup_of_a_billion_ids():
    from paper_2605_15695_amd.embedding import embedding

    n, d = 1 << 30, 49
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < n * (4 * d + 8) + (4 << 30):
        pytest.skip("not enough free memory for 210 GB of rows")
    table = torch.randn(7, d, generator=_gen(1), device="cuda")
    ids = torch.empty(n, dtype=torch.int32, device="cuda")
    ids.view(-1, 1 << 20).copy_((torch.arange(1 << 20, device="cuda") % 8).to(torch.int32))  # 7: no row
    out = embedding(ids, table, 2.0)
    want = torch.cat([table * 2.0, torch.zeros(1, d, device="cuda")]).repeat(1 << 17, 1)  # of 2^20 ids
    try:
        for at in range(0, n, 1 << 20):
            assert torch.equal(out[at:at + (1 << 20)], want), at
    finally:
        del out, ids, want
        torch.cuda.empty_cache()


# rows without an id: +0, whatever the scale, by each way their zeros are written
@pytest.mark.parametrize("n,rows,d", [(50, 20, 5), (50, 3000, 5), (1000, 600, 64), (5000, 9000, 5), (20000, 30000, 5)])
@pytest.mark.parametrize("scale", [-2.0, float("inf"), float("nan")])
def test_rows_without_ids_do_not_know_the_scale(path, n, rows, d, scale):
    from paper_2605_15695_amd.embedding import embedding

    ids = torch.randint(0, rows // 2, (n,), generator=_gen(n), device="cuda") * 2 + 1
    table = torch.ones(rows, d, device="cuda").requires_grad_()
    grad, = torch.autograd.grad(embedding(ids, table, scale), table, torch.ones(n, d, device="cuda"))
    met = torch.zeros(rows, dtype=torch.bool, device="cuda")
    met[ids] = True
    assert not bool(grad[~met].view(torch.int32).any())  # all bits 0
    want = torch.bincount(ids, minlength=rows)[met].float()[:, None].expand(-1, d) * scale
    assert torch.equal(grad[met].nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))


# forward-mode derivatives: there are none, and a call says so
def test_tangents_are_refused(path):
    import torch.autograd.forward_ad as fw

    from paper_2605_15695_amd.embedding import embedding
    from paper_2605_15695_amd.muon import orthogonalize
    from paper_2605_15695_amd.norm import group_norm

    X, w, b = torch.randn(10, 8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    ids, off = torch.tensor([0, 3, 3], device="cuda"), torch.tensor([0, 4, 10], device="cuda")
    calls = [(lambda t: embedding(ids, t), X), (lambda t: group_norm(t, 2), X), (lambda t: group_norm(t, 2, w, b, off, activation="silu"), X),
             (lambda t: group_norm(X, 2, t, b), w), (lambda t: group_norm(X, 2, None, t), b), (orthogonalize, X),
             (lambda t: orthogonalize(t.view(2, 5, 8)), X)]
    for call, at in calls:
        for leaf in (at, at.clone().requires_grad_()):
            want = call(leaf)
            with fw.dual_level():
                dual = fw.make_dual(leaf, torch.ones_like(leaf))
                with pytest.raises(NotImplementedError):
                    call(dual)
                with torch.no_grad(), pytest.raises(NotImplementedError):
                    call(dual)
                assert torch.equal(call(leaf), want)  # without one
    with fw.dual_level():  # a dual number whose primal lies elsewhere, and empty inputs
        with pytest.raises(NotImplementedError):
            group_norm(fw.make_dual(X[:0], X[:0]), 2)
        with pytest.raises(NotImplementedError):
            orthogonalize(fw.make_dual(X.t(), X.t()))


def test_an_orthogonalised_matrix_is_a_constant(path):
    from paper_2605_15695_amd.muon import orthogonalize

    assert not orthogonalize(torch.randn(4, 5, device="cuda").requires_grad_()).requires_grad


# a view whose numbers are stored with the other sign
def test_views_with_a_sign(path):
    from paper_2605_15695_amd.embedding import embedding
    from paper_2605_15695_amd.muon import Muon, orthogonalize
    from paper_2605_15695_amd.norm import group_norm

    z = torch.randn(30, 1, generator=_gen(2), device="cuda", dtype=torch.complex64)
    wide = torch.randn(30, 8, generator=_gen(3), device="cuda")
    ids = torch.tensor([3, -1, 29], device="cuda")
    for t in (z.conj().imag, torch._neg_view(wide)):
        assert t.is_neg()
        plain = t.resolve_neg().clone()
        assert not plain.is_neg()
        assert torch.equal(embedding(ids, t), embedding(ids, plain))
        assert torch.equal(group_norm(t, 1), group_norm(plain, 1))
        assert torch.equal(orthogonalize(t), orthogonalize(plain))
        w, signed = plain[0].contiguous(), torch._neg_view(-plain[0])
        assert signed.is_neg()
        assert torch.equal(group_norm(plain, 1, signed, signed), group_norm(plain, 1, w, w))
        grads = []
        for g in (t, plain):
            x = plain.clone().requires_grad_()
            p = torch.nn.Parameter(plain.clone())
            p.grad = g
            opt = Muon([p])
            opt.step()
            opt.step()
            grads.append([*torch.autograd.grad(embedding(torch.arange(30, device="cuda"), x), x, g), *torch.autograd.grad(group_norm(x, 1), x, g), p.detach()])
        assert all(torch.equal(a, b) for a, b in zip(*grads))


# the distance of rows means nothing where there is one
def test_one_row_at_any_distance(path):
    from paper_2605_15695_amd.embedding import embedding
    from paper_2605_15695_amd.muon import Muon, orthogonalize
    from paper_2605_15695_amd.norm import group_norm

    row = torch.randn(1, 40, generator=_gen(1), device="cuda")
    far = row.as_strided((1, 40), ((1 << 31) + 8, 1))
    ids = torch.tensor([0, 0, -1], device="cuda")
    assert torch.equal(embedding(ids, far), embedding(ids, row))
    assert torch.equal(group_norm(far, 4), group_norm(row, 4))
    assert torch.equal(orthogonalize(far), orthogonalize(row))
    out = []
    for g in (row, far):
        x, p = row.clone().requires_grad_(), torch.nn.Parameter(row.clone().as_strided(g.shape, g.stride()))
        grads = torch.autograd.grad(embedding(ids[:1], x), x, g) + torch.autograd.grad(group_norm(x, 4), x, g)
        p.grad, opt = g, Muon([p])
        opt.step()
        opt.step()
        out.append([*grads, p.detach()])
    assert all(torch.equal(a, b) for a, b in zip(*out))


# sizes that the library refuses: the same exception with the same code by either path, with and without a gradient to come
def test_refusals_of_the_library_are_one_exception(path):
    import paper_2605_15695_amd as pc
    from paper_2605_15695_amd.embedding import embedding
    from paper_2605_15695_amd.norm import group_norm

    ids = torch.zeros(1, dtype=torch.int64, device="cuda")
    table = torch.zeros(1, (1 << 23) + 1, device="cuda")  # wider than a table may be
    X = torch.zeros(1, (1 << 22) + 2048, device="cuda")   # more channels than there may be
    for call, t in ((lambda t: embedding(ids, t), table), (lambda t: group_norm(t, 2049), X)):
        for leaf in (t, t.clone().requires_grad_()):
            with pytest.raises(pc.PcsrError) as e:
                call(leaf)
            assert e.value.code == pc.binding.PCSR_E_TOO_LARGE


def test_refusals_in_a_backward_pass_are_the_same_exception(path):
    import paper_2605_15695_amd as pc
    from paper_2605_15695_amd.embedding import embedding

    # a gradient whose rows lie further apart than the library takes: one long row of another array
    ids = torch.zeros(2, dtype=torch.int64, device="cuda")
    table = torch.zeros(3, 2, device="cuda", dtype=torch.bfloat16).requires_grad_()
    far = torch.zeros((1 << 31) + 16, device="cuda", dtype=torch.bfloat16).as_strided((2, 2), ((1 << 31) + 8, 1))
    out = embedding(ids, table)
    with pytest.raises(pc.PcsrError) as e:
        torch.autograd.grad(out, table, far)
    assert e.value.code == pc.binding.PCSR_E_TOO_LARGE


# more matrices than fit any array of fixed size
@pytest.mark.parametrize("shape", [(4097, 3, 5), (5000, 8, 8)])
def test_thousands_of_matrices(path, shape):
    from paper_2605_15695_amd.muon import orthogonalize

    G = torch.randn(*shape, generator=_gen(4), device="cuda")
    out = orthogonalize(G)
    for at in (0, 23, 24, 4095, 4096, shape[0] - 1):
        assert torch.equal(out[at], orthogonalize(G[at]))


def test_a_step_of_thousands_of_matrices(path):
    from paper_2605_15695_amd.muon import Muon

    g = _gen(5)
    shapes = [(2, 3), (4, 2), (130, 2), (1, 1)] * 1030  # 1030 of them too wide for the launch of small ones
    params = [torch.nn.Parameter(torch.zeros(s, device="cuda")) for s in shapes]
    for p in params:
        p.grad = torch.randn(p.shape, generator=g, device="cuda")
    opt = Muon(params, lr=0.1)
    opt.step()
    opt.step()  # not the first step
    for at in (0, 1, 2, 3, 4094, 4097, 4098, len(shapes) - 1):
        p = torch.nn.Parameter(torch.zeros(shapes[at], device="cuda"))
        p.grad = params[at].grad
        opt = Muon([p], lr=0.1)
        opt.step()
        opt.step()
        assert torch.equal(p, params[at])


# A weight of 0 leaves the bias: gelu and its slope at chosen places.  With u = 2^-24 the exponential of -z^2/2 is off by 1.2 z^2 u (its
# argument is rounded twice) and 2 u, the share below z by the polynomial's 3e-8 and some ten roundings beside it, so 16 u; where z is
# positive a difference from 1 makes these absolute.
def test_gelu_keeps_its_digits_far_below_zero(path):
    from paper_2605_15695_amd.norm import group_norm

    z = torch.cat([torch.linspace(-12.5, 6.0, 40_000, device="cuda"), torch.zeros(1, device="cuda")])
    C = z.numel()
    x = torch.zeros(1, C, device="cuda").requires_grad_()
    w, b = torch.zeros(C, device="cuda"), z.clone().requires_grad_()
    y = group_norm(x, C, w, b, activation="gelu")
    slope, = torch.autograd.grad(y, b, torch.ones_like(y))
    z = z.double()
    below, bell = 0.5 * torch.erfc(-z / 2.0 ** 0.5), torch.exp(-0.5 * z * z) / (2.0 * torch.pi) ** 0.5
    size = torch.minimum(below, torch.erfc(z / 2.0 ** 0.5) * 0.5) * (16 + 2 * z * z) + below * (z > 0) * 2
    tiny = 2.0 ** -126  # numbers without a leading bit may be zeros
    assert bool(((y.detach().double()[0] - z * below).abs() <= U * (z.abs() * size + (z * below).abs()) + tiny).all())
    assert bool(((slope.double() - below - z * bell).abs() <= U * (size + z.abs() * bell * (8 + 2 * z * z) + below + z.abs() * bell) + tiny).all())


# polynomials that first make singular values small: products of small numbers keep their bits too.  The second step takes s = 1e-6 to s (1 - 0.5 + 0.1)
@pytest.mark.parametrize("shape", [(30, 50), (300, 170)])
def test_polynomials_that_shrink_first(shape):
    from paper_2605_15695_amd.muon import orthogonalize
    from test_gpu_muon import BOUND, _near, _polynomial

    # one strong direction: X has a singular value of nearly 1
    G = torch.randn(shape[0], 1, generator=_gen(1), device="cuda") @ torch.randn(1, shape[1], generator=_gen(2), device="cuda")
    G += 0.01 * torch.randn(*shape, generator=_gen(3), device="cuda")
    for small in (1e-3, 1e-6, 1e-9):
        steps = [(small, 0.0, 0.0), (1.0, -0.5 / small ** 2, 0.1 / small ** 4)]
        _near(orthogonalize(G, 2, steps), _polynomial(G, 2, tuple(steps)), BOUND[torch.float32])
