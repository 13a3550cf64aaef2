"""The instances of the kernels around the graph layers that large calls take: gradients of a table by sorted ids in rows of many
pieces, products in tiles of 128, teams of a wavefront with whole groups to a thread; by the checks (and with the tolerances)
of the tests of each operator."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_gpu_embedding as embed  # noqa: E402
import test_gpu_muon as muon  # noqa: E402
import test_gpu_norm as norm  # noqa: E402


# ids sorted by ranks (up to 16,384) and by passes; 4 to 64 lanes to a row, rows of one slice and of several
@pytest.mark.parametrize("kind", list(embed.TYPES))
@pytest.mark.parametrize("n", [4500, 16384, 20000])
@pytest.mark.parametrize("rows,d,how", [(3000, 1000, "skewed"), (70000, 250, "outside"), (40, 260, "any"), (6, 515, "any"), (900, 2051, "skewed"),
                                        (5000, 128, "any"), (5, 128, "one"), (3000, 203, "outside"), (20000, 67, "skewed"), (300, 30, "any")])
def test_wide_rows_by_sorted_ids(kind, n, rows, d, how):
    g = embed._gen(n + rows + d)
    ids = embed._ids(g, n, rows, how)
    table = torch.randn(rows, d, generator=g, device="cuda").to(embed.TYPES[kind][0])
    dout = torch.randn(n, d, generator=g, device="cuda").to(embed.TYPES[kind][0])
    embed._check(ids if d % 2 else ids.to(torch.int32), table, dout, 0.7, kind)


# 16 bits, hundreds of thousands of ids
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n,rows,d", [(300_000, 1 << 20, 24), (150_000, 2000, 65)])
def test_many_ids_of_16_bits(kind, n, rows, d):
    g = embed._gen(n)
    ids = embed._ids(g, n, rows, "skewed")
    table = torch.randn(rows, d, generator=g, device="cuda").to(embed.TYPES[kind][0])
    embed._check(ids, table, torch.randn(n, d, generator=g, device="cuda").to(embed.TYPES[kind][0]), 1.5, kind)


def _space(m, n, tile):
    """Workspace of a matrix of m <= n, in bytes: planes of X, of its transpose twice, of A and B, X and A in fp32"""
    M, N = -(-m // tile) * tile, -(-n // tile) * tile
    return 3 * 2 * 2 * M * N + 2 * 2 * 2 * M * M + 4 * M * N + 4 * M * M  # two fp16 numbers each


def _check_tiles(shape, kind, tile):
    """That a call of these matrices asks for the workspace that tiles of that size need"""
    import ctypes

    from paper_2605_15695_amd import binding as pc

    count, rows, cols = shape if len(shape) == 3 else (1, *shape)
    lo, hi = min(rows, cols), max(rows, cols)
    many = (pc.pcsr_matrix_t * count)(*[pc.pcsr_matrix_t(4096, None, 4096, rows, cols, cols, 0, cols, 0.0, 0)] * count)
    co = (ctypes.c_double * 15)(*muon.QUINTIC * 5)
    number = [torch.float32, torch.bfloat16, torch.float16].index(kind)
    how = pc.pcsr_ortho_t(number, 5, ctypes.addressof(co), 0, 0, 0.0, 0.0)
    have = pc._lib().pcsr_ortho_workspace(many, count, ctypes.byref(how)) - 24 * 256 * 8
    sizes = {t: count * _space(lo, hi, t) for t in (64, 128)}
    assert have == sizes[tile] and sizes[64] != sizes[128], (have, sizes)


# sides that are no whole tiles, both ways round, one matrix and several
@pytest.mark.parametrize("dtype", muon.TYPES)
@pytest.mark.parametrize("shape,tile", [((1930, 2100), 128), ((2430, 1970), 128), ((4, 910, 1030), 128), ((5, 1200, 780), 128), ((13, 1000, 1030), 128),
                                        ((1100, 1700), 64), ((3, 780, 910), 64)])
def test_large_tiles(dtype, shape, tile):
    from paper_2605_15695_amd.muon import orthogonalize

    _check_tiles(shape, dtype, tile)
    G = torch.randn(*shape, generator=muon._gen(sum(shape)), device="cuda").to(dtype)
    out = orthogonalize(G)
    assert torch.equal(out, orthogonalize(G))
    for g, o in zip(G if G.dim() == 3 else G[None], out if G.dim() == 3 else out[None]):
        muon._near(o, muon._polynomial(g), muon.BOUND[dtype])


# a step of matrices that take tiles of 128, with momentum and strides
@pytest.mark.parametrize("dtype", muon.TYPES)
@pytest.mark.parametrize("shape,count", [((1000, 900), 4), ((770, 1030), 13)])
def test_steps_of_large_matrices(dtype, shape, count):
    from paper_2605_15695_amd.muon import Muon

    g = muon._gen(6)
    big = [torch.randn(shape[0], shape[1] + 7, generator=g, device="cuda").to(dtype) for _ in range(count)]
    params = [torch.nn.Parameter(t[:, 3:3 + shape[1]]) for t in big]
    opt, lr = Muon(params, lr=0.1, weight_decay=0.1), 0.1
    bufs = [torch.zeros(shape, device="cuda", dtype=torch.float64) for _ in params]
    u = {torch.float32: 2.0 ** -23, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    for _ in range(2):
        was = [p.detach().double() for p in params]
        edges = [(t[:, :3].clone(), t[:, 3 + shape[1]:].clone()) for t in big]
        for p in params:
            p.grad = torch.randn(shape, generator=g, device="cuda").to(dtype)
        opt.step()
        for k, (p, w) in enumerate(zip(params, was)):
            bufs[k] = 0.95 * bufs[k] + p.grad.double()
            O = muon._polynomial(p.grad.double() + 0.95 * bufs[k])
            gain = max(1.0, shape[0] / shape[1]) ** 0.5
            want = w * (1.0 - lr * 0.1) - lr * gain * O
            off = float((p.detach().double() - want).norm())
            assert off <= muon.BOUND[dtype] * lr * gain * float(O.norm()) + u * float(want.norm()), (k, off)
        for t, (a, b) in zip(big, edges):
            assert torch.equal(t[:, :3], a) and torch.equal(t[:, 3 + shape[1]:], b)


# teams of a wavefront (512 graphs and more, a few kilobytes each on the average): whole groups to a thread, and not; graphs that a team keeps, reads
# again, and leaves to the chunks
@pytest.mark.parametrize("kind,act", [("fp32", "gelu"), ("bf16", "silu"), ("bf16", "relu"), ("fp16", "gelu"), ("fp16", "none")])
@pytest.mark.parametrize("C,groups", [(64, 8), (256, 2), (64, 1), (512, 1), (40, 5), (24, 24), (36, 3), (200, 8)])
@pytest.mark.parametrize("lengths", [[8] * 700 + [0] * 5 + [2000], [1 + k % 5 for k in range(900)] + [300, 0, 90]])
def test_teams_of_a_wavefront(kind, act, C, groups, lengths):
    X, w, b = norm._inputs(sum(lengths) + C, sum(lengths), C, kind)
    norm._check(X, groups, w, b, lengths, norm._offsets(lengths, C % 3 == 0), act, kind)
