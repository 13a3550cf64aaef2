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
