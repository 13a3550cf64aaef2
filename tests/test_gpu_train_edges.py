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
