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
                                  (16_384, 32, 768), (512, 320, 2048), (131_072, 64, 256), (140_001, 8, 40)], ids=lambda s: "x".join(map(str, s)))
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


# Slopes as they are kept for 16-bit types: within 2^-16, and those below zero, which become small far out, within 2^-10 of themselves down to 2^-45.  Beside that an
# activation's own arithmetic: with s = p + z q, p the share below z and z q the other term, of which roundings take up to 16 U (1 + z^2) or 16 U (1 + |z|)
# of both; gelu's share of 16-bit types is good to 2^-14 of what it is below zero, and above zero of what is left to 1.
def _slopes(z, act):
    """slope and what it may be off by beside the way it is kept"""
    U = 2.0 ** -24
    if act == "silu":
        p, left = torch.sigmoid(z), torch.sigmoid(-z)
        return p * (1 + z * left), 16 * U * (1 + z.abs()) * p * (1 + z.abs() * left)
    p, left = 0.5 * torch.erfc(-z / 2.0 ** 0.5), 0.5 * torch.erfc(z / 2.0 ** 0.5)
    q = torch.exp(-0.5 * z * z) / (2 * torch.pi) ** 0.5
    return p + z * q, 16 * U * (1 + z * z) * (p + z.abs() * q) + 2.0 ** -14 * torch.minimum(p, left)


def _taken(code):
    """16 bits as pcsr_train.h describes them"""
    code = code.long() & 0xFFFF
    small = (((code - 45312) << 14) + 0xA9000000) & 0xFFFFFFFF
    small = torch.where(small >= 1 << 31, small - (1 << 32), small).int().view(torch.float32).double()
    return torch.where(code >= 45312, small, torch.where(code == 0, torch.nan, code.double() / 32768 - 0.25))


def _kept_within(s, own):
    half = 2.0 ** -16 + 2.0 ** -23
    return torch.where(s < 0, torch.minimum(torch.full_like(s, half), s.abs() * 2.0 ** -10), torch.full_like(s, half)) * (1 + 2.0 ** -12) + own * (1 + 2.0 ** -9) + 2.0 ** -45


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 8, 20, 600, 33_000])  # few of them, tiles, weights in LDS
def test_kept_slopes(kind, act, rows):
    from paper_2605_15695_amd import binding as pc

    N, K = 512, 32
    lib = pc._lib()
    X, W = torch.zeros(rows, K, device="cuda", dtype=TYPES[kind][0]), torch.zeros(N, K, device="cuda", dtype=TYPES[kind][0])
    y = torch.empty(rows, N, device="cuda", dtype=TYPES[kind][0])
    for lo, hi in ((-36.0, -12.0), (-12.0, -4.0), (-4.0, 0.0), (-1.3, -1.25), (-0.8, -0.7), (0.0, 8.0), (8.0, 60.0)):
        b = torch.linspace(lo, hi, N, device="cuda")
        code = torch.zeros(rows, N, dtype=torch.int16, device="cuda")
        a = pc.pcsr_linear_t(rows, K, N, NUMBERS[kind], 0, {"silu": 2, "gelu": 3}[act], 0, X.data_ptr(), W.data_ptr(), b.data_ptr(), None, K, K, 0,
                             pc.pcsr_drop_t(0.0, 0, 0, None, None))
        ws = torch.empty(lib.pcsr_linear_workspace(ctypes.byref(a), 0) + 16, dtype=torch.uint8, device="cuda")
        assert lib.pcsr_linear(ctypes.byref(a), y.data_ptr(), code.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream) == pc.PCSR_OK
        s, own = _slopes(b.double(), act)
        far = (_taken(code) - s).abs() - _kept_within(s, own)
        assert bool((far <= 0).all()), (lo, hi, float(far.max()))


# In all: gelu's arithmetic for 16-bit types adds up to 1.15 2^-16 (the degree 4 share at 0, by its polynomial in 64 bits), fp32 roundings 64 U at most where slopes are not small.
@pytest.mark.parametrize("act,most", [("relu", 0.0), ("silu", 2.0 ** -16), ("gelu", 2.15 * 2.0 ** -16)])
def test_kept_slopes_in_all(act, most):
    from paper_2605_15695_amd import binding as pc

    N, K = 4096, 8
    X, W = torch.zeros(1, K, device="cuda", dtype=torch.float16), torch.zeros(N, K, device="cuda", dtype=torch.float16)
    y, code, b = torch.empty(1, N, device="cuda", dtype=torch.float16), torch.zeros(1, N, dtype=torch.int16, device="cuda"), torch.linspace(-8.0, 8.0, N, device="cuda")
    b[N // 2] = 0.0
    a = pc.pcsr_linear_t(1, K, N, 2, 0, {"relu": 1, "silu": 2, "gelu": 3}[act], 0, X.data_ptr(), W.data_ptr(), b.data_ptr(), None, K, K, 0, pc.pcsr_drop_t(0.0, 0, 0, None, None))
    assert pc._lib().pcsr_linear(ctypes.byref(a), y.data_ptr(), code.data_ptr(), None, torch.cuda.current_stream().cuda_stream) == pc.PCSR_OK
    s = (b > 0).double() if act == "relu" else _slopes(b.double(), act)[0]
    far = (_taken(code)[0] - s).abs().max()
    assert float(far) <= most + (64 * 2.0 ** -24 if act != "relu" else 0.0)


# units whose sums are all far below zero: their gradients are small, not none.  dz = s dy is rounded to the type (fp16: 2^-25 where it is small).
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [5, 300, 5000, 131_072])
def test_gradients_of_small_slopes(kind, act, rows):
    from paper_2605_15695_amd.linear import linear

    N = 64
    u, dtype = TYPES[kind][1], TYPES[kind][0]
    X, W = torch.zeros(rows, N, device="cuda", dtype=dtype, requires_grad=True), torch.eye(N, device="cuda", dtype=dtype)
    b = torch.linspace(-20.0 if act == "silu" else -6.0, -2.0, N, device="cuda").requires_grad_()
    dy = torch.full((rows, N), 2.0 ** 15, device="cuda", dtype=dtype)
    dx, db = torch.autograd.grad(linear(X, W, b, act), (X, b), dy)
    s, own = _slopes(b.detach().double(), act)
    off = _kept_within(s, own)
    assert bool(((dx.double() - 2.0 ** 15 * s).abs() <= 2.0 ** 15 * (off * (1 + u) + 2 * u * s.abs()) + 2.0 ** -23).all())
    assert bool(((db.double() - rows * 2.0 ** 15 * s).abs() <= rows * 2.0 ** 15 * (off + 140 * 2.0 ** -24 * s.abs())).all())


# fp32 numbers out of the pieces' range in a backward pass: the tiles that meet them are done again as products of fp32 numbers, K roundings one after the other, and multiplied by
# 1 / (1 - p) like the others (small tiles side by side, rows past weights in LDS, weights in planes, both operands in pieces)
@pytest.mark.parametrize("size", [(200, 96, 70), (40_000, 24, 40), (50_000, 300, 300), (20, 3000, 40)], ids=lambda s: "x".join(map(str, s)))
def test_range_behind_dropout(size):
    from drop_reference import kept
    from paper_2605_15695_amd.linear import linear

    M, K, N = size
    U, p = 2.0 ** -24, 0.25
    X, W, dy = _normal(21, M, K), _normal(22, N, K), _normal(23, M, N)
    W[N - 1, K - 1], X[M - 1, 0], dy[M // 2, N // 2] = 2.0 ** 60, 2.0 ** 50, -2.0 ** 40
    k, f = kept(M, N, p, 4, 3)
    g = torch.from_numpy(k).cuda().double() * f * dy.double()
    X.requires_grad_(), W.requires_grad_()
    dx, dw = torch.autograd.grad(linear(X, W, p=p, seed=4, offset=3), (X, W), dy)
    for got, a, b, n in ((dx, g, W.detach().double(), N), (dw, g.t(), X.detach().double(), M)):
        err = (n + 4) * U * (a.abs() @ b.abs())
        assert bool(((got.double() - a @ b).abs() <= err + 2.0 ** -120).all())
