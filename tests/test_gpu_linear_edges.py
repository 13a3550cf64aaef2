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
