"""Linear layers where workspaces, slopes and ranges end, against the formulas in 64 bits: see test_gpu_linear.py for what results may be off by."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_linear import TYPES, _normal, check  # noqa: E402

NUMBERS = {"fp32": 0, "bf16": 1, "fp16": 2}
BAND = 16 << 20


# What lies behind a workspace of the size that is asked for is as it was: sums of stretches are as long as the way that runs makes them, however operands lie.
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("size", [(12_288, 192, 192), (18_432, 128, 192), (8286, 152, 176), (22_528, 64, 320), (2048, 512, 320), (8192, 160, 160),
                                  (16_384, 32, 768), (512, 320, 2048)], ids=lambda s: "x".join(map(str, s)))
def test_nothing_behind_the_workspace(kind, size):
    from paper_2605_15695_amd import binding as pc

    M, K, N = size
    X, W, dy = _normal(1, M, K, kind=kind), _normal(2, N, K, kind=kind, scale=K ** -0.5), _normal(3, M, N, kind=kind)
    dx, dw, db = torch.empty_like(X), torch.empty_like(W), torch.empty(N, device="cuda")
    a = pc.pcsr_linear_t(M, K, N, NUMBERS[kind], 0, 0, 0, X.data_ptr(), W.data_ptr(), None, None, K, K, 0, pc.pcsr_drop_t(0.0, 0, 0, None, None))
    lib = pc._lib()
    need, ends = lib.pcsr_linear_workspace(ctypes.byref(a), 1), (ctypes.c_int64 * 8)()
    assert lib.pcsr_linear_uses(ctypes.byref(a), dy.data_ptr(), N, ends) == pc.PCSR_OK and max(ends) <= need
    room = torch.full((need + BAND,), 0xA5, dtype=torch.uint8, device="cuda")
    for which in ((dx, dw, db), (None, dw, None), (dx, None, None)):
        room[:need].fill_(0xFF)  # (not a number, read as fp32)
        rc = lib.pcsr_linear_backward(ctypes.byref(a), None, dy.data_ptr(), N, *(None if t is None else t.data_ptr() for t in which), room.data_ptr(),
                                      torch.cuda.current_stream().cuda_stream)
        assert rc == pc.PCSR_OK and bool((room[need:] == 0xA5).all())
        check(X, W, torch.zeros(N, device="cuda"), "none", None, 0.0, 0, 0, kind, dy, grads=(dx, dw, db))


# 1 / (1 - p) multiplies what the gradient's products add up to: fp16 gradients near its last number, 65,504, stay numbers, whatever kernels come by (small tiles side
# by side, any operands, straight ones, rows past weights in LDS, one read).  With no activation, or relu, the gradient at z is dy's numbers or none: then only results are rounded.
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("act,p", [("none", 0.5), ("relu", 0.875), ("silu", 0.75)])
@pytest.mark.parametrize("size", [(20, 8, 16), (777, 75, 333), (512, 1024, 512), (4100, 520, 1032), (33_000, 64, 96), (40_000, 301, 260), (131_072, 64, 64), (131_100, 24, 200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_large_gradients_behind_dropout(kind, size, act, p):
    from paper_2605_15695_amd.linear import linear

    M, K, N = size
    X, W = _normal(11, M, K, kind=kind, scale=2.0 ** -13), _normal(12, N, K, kind=kind, scale=2.0 ** -11)
    b = _normal(13, N)
    dy = (_normal(14, M, N).sign() * (30_000 + 1000 * _normal(15, M, N))).clamp(-36_000, 36_000).to(TYPES[kind][0])
    leaves = [t.requires_grad_() for t in (X, W, b)]
    grads = torch.autograd.grad(linear(X, W, b, act, None, p, 5, 1), leaves, dy)
    assert all(bool(g.isfinite().all()) for g in grads)
    check(X, W, b, act, None, p, 5, 1, kind, dy, grads=grads)
    if act == "silu" or kind == "fp32":
        return
    u, U = TYPES[kind][1], 2.0 ** -24  # the bound without a rounding of dz
    from drop_reference import kept

    k, f = kept(M, N, p, 5, 1)
    g = torch.from_numpy(k).cuda().double() * f * dy.double()
    z = X.detach().double() @ W.detach().double().t() + b.detach().double()
    if act == "relu":
        assert float(z.abs().min()) > 1e-9  # (z is off by less: X W^T is below 2^-14)
        g = g * (z > 0)
    for got, want, size_of, n in ((grads[0], g @ W.detach().double(), g.abs() @ W.detach().double().abs(), N),
                                  (grads[1], g.t() @ X.detach().double(), g.abs().t() @ X.detach().double().abs(), M)):
        err = ((n / 8 + 51) * U * size_of) * (1 + u) + u * want.abs() + 2.0 ** -24
        assert bool(((got.double() - want).abs() <= err).all())
