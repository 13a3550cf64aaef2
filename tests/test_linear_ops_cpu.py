"""Dropout and linear layers without a GPU: the generator against its published values, what the C entry points and the Python calls refuse
before they touch the device."""
import ctypes

import numpy as np
import pytest

from drop_reference import kept, philox
from paper_2605_15695_amd import binding as pc

torch = pytest.importorskip("torch")

OK, INVALID, UNSUPPORTED, TOO_LARGE = pc.PCSR_OK, pc.PCSR_E_INVALID_ARG, pc.PCSR_E_UNSUPPORTED, pc.PCSR_E_TOO_LARGE
P = 4096  # an address: nothing is read there


# the known answers that the generator was published with
@pytest.mark.parametrize("counter,key,words", [
    ([0] * 4, [0] * 2, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], "d16cfe09 94fdcceb 5001e420 24126ea1")])
def test_reference_generator(counter, key, words):
    assert " ".join("%08x" % int(w) for w in philox(counter, key)) == words


def test_reference_places():
    k, f = kept(3, 19, 0.25, 5, 1 << 33)
    words = philox([2, 1, 0, 2], [5, 0])
    bits = [h for w in words for h in (int(w) & 0xFFFF, int(w) >> 16)]
    assert k[1, 16:].tolist() == [b >= 16384 for b in bits[:3]] and f == 65536 / 49152
    assert np.array_equal(kept(1, 19, 0.25, 5, 1 << 33, first=2)[0], k[2:])
    assert not kept(4, 4, 1.0, 1, 1)[0].any() and kept(4, 4, 0.0, 1, 1)[0].all()


def test_dropout_entry_point():
    lib = pc._lib()

    def call(rows=3, cols=4, type=0, x=P, x_stride=4, residual=None, r_stride=0, p=0.5, out=P, how=True):
        d = pc.pcsr_drop_t(p, 1, 2, None, None)
        return lib.pcsr_dropout(rows, cols, type, x, x_stride, residual, r_stride, ctypes.byref(d) if how else None, out, None)

    for bad in (dict(rows=-1), dict(cols=0), dict(x=None), dict(out=None), dict(x_stride=3), dict(residual=P, r_stride=3), dict(p=-0.1), dict(p=1.1),
                dict(p=float("nan")), dict(how=False)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(type=3), dict(type=-1)):
        assert call(**bad) == UNSUPPORTED
    for bad in (dict(rows=1 << 32), dict(cols=1 << 31, x_stride=1 << 31)):
        assert call(**bad) == TOO_LARGE
    assert call(rows=0, x=None, out=None) == OK


def _linear(**kw):
    a = pc.pcsr_linear_t(10, 12, 14, 0, 0, 0, 0, P, P, None, None, 12, 12, 14, pc.pcsr_drop_t(0.0, 0, 0, None, None))
    for k, v in kw.items():
        if k == "p":
            a.drop.p = v
        else:
            setattr(a, k, v)
    return a


def test_linear_entry_points():
    lib = pc._lib()

    def fwd(y=P, z=None, ws=P, **kw):
        return lib.pcsr_linear(ctypes.byref(_linear(**kw)), y, z, ws, None)

    def bwd(z=P, dy=P, stride=14, dx=P, dw=P, db=P, ws=P, **kw):
        return lib.pcsr_linear_backward(ctypes.byref(_linear(**kw)), z, dy, stride, dx, dw, db, ws, None)

    for call in (fwd, bwd):
        for bad in (dict(rows=-1), {"in": -1}, dict(out=0), dict(x_stride=11), dict(w_stride=11), dict(x=None), dict(w=None), dict(p=2.0),
                    dict(p=float("nan"))):
            assert call(**bad) == INVALID, bad
        for bad in (dict(type=3), dict(type=-1), dict(act=4), dict(act=-1), dict(bias_type=1), dict(type=1, bias_type=2)):
            assert call(**bad) == UNSUPPORTED, bad
        # tiles of 64 x 64 past 2^23: 2^18 rows of 2^17 and more, and too many rows and columns
        for bad in (dict(rows=(1 << 18) + 1, out=1 << 17), dict(rows=1 << 32), dict(out=1 << 24), {"in": 1 << 24, "x_stride": 1 << 24, "w_stride": 1 << 24},
                    {"out": 1 << 20, "in": 1 << 20, "x_stride": 1 << 20, "w_stride": 1 << 20}):
            assert call(**bad) == TOO_LARGE, bad
    assert fwd(y=None) == INVALID and fwd(residual=P, r_stride=13) == INVALID and fwd(rows=0, y=None, x=None) == OK
    assert bwd(dy=None) == INVALID and bwd(stride=13) == INVALID and bwd(ws=None) == INVALID and bwd(act=2, z=None) == INVALID
    assert bwd(dx=None, dw=None, db=None) == OK and bwd(rows=0, dy=None) == OK
    deep = _linear(rows=100, **{"in": 100_000, "x_stride": 100_000, "w_stride": 100_000})
    assert lib.pcsr_linear_workspace(ctypes.byref(deep), 0) > 0 and lib.pcsr_linear(ctypes.byref(deep), P, None, None, None) == INVALID
    assert lib.pcsr_linear_workspace(None, 0) == 0 and lib.pcsr_linear(None, P, None, P, None) == INVALID


# what a backward pass writes of its workspace lies within what is asked for, however its operands lie: each part behind the one before
def _parts(rows, cols_in, out, kind, act=0, odd=(0, 0, 0), p=0.0):
    """bytes asked for, and (first, last) of the four parts that are written; odd: of x, w and dy, whether they lie at odd addresses"""
    size = 2 if kind else 4
    a = _linear(rows=rows, out=out, type=kind, act=act, x_stride=cols_in, w_stride=cols_in, x=P + size * odd[0], w=P + size * odd[1], p=p, **{"in": cols_in})
    ends = (ctypes.c_int64 * 8)()
    assert pc._lib().pcsr_linear_uses(ctypes.byref(a), P + size * odd[2], out, ends) == OK
    return pc._lib().pcsr_linear_workspace(ctypes.byref(a), 1), [(ends[2 * k], ends[2 * k + 1]) for k in range(4)]


def _fits(*case, **kw):
    asked, parts = _parts(*case, **kw)
    at = 0
    for first, last in parts:
        assert at <= first <= last and first % 16 == 0, (case, kw, asked, parts)
        at = last
    assert at <= asked, (case, kw, asked, parts)
    return asked, parts


LYING = [(x, w, dy) for x in (0, 1) for w in (0, 1) for dy in (0, 1)]


@pytest.mark.parametrize("size", [(12_288, 192, 192), (18_432, 128, 192), (8286, 152, 176), (22_528, 64, 320), (2048, 512, 320), (8192, 160, 160),
                                  (16_384, 32, 768), (512, 320, 2048), (480_000, 64, 256), (777, 75, 333), (1, 1, 1), (131_072, 8, 8), (40, 0, 9)],
                         ids=lambda s: "x".join(map(str, s)))
def test_workspace_of_a_backward_pass(size):
    for kind in (0, 1, 2):
        for odd in LYING:
            for kw in (dict(), dict(act=2), dict(p=0.5)):
                _fits(*size, kind, odd=odd, **kw)


def test_workspace_of_many_sizes():
    rng = np.random.default_rng(11)
    for n in range(30_000):
        M, K, N = (int(np.exp(v)) for v in rng.uniform(0, (13.5, 8.5, 8.5)))
        if n % 4:  # whole pieces of 16 bytes, as a model's widths are: operands that can lie either way
            K, N = -(-K // 8) * 8, -(-N // 8) * 8
        if -(-K // 64) * -(-N // 64) > 1 << 23:
            continue
        for kind in (n % 2 + 1, 0) if n % 3 == 0 else (n % 2 + 1,):
            for odd in LYING[:4:2] + LYING[4:6]:
                _fits(M, K, N, kind, odd=odd, act=2 * (n % 5 == 0))


# one read for all gradients: sums of its 256 workgroups and nothing else
@pytest.mark.parametrize("size", [(480_000, 64, 256), (131_072, 8, 8), (2_000_000, 64, 64)], ids=lambda s: "x".join(map(str, s)))
def test_workspace_of_one_read(size):
    M, K, N = size
    for kind in (1, 2):
        for kw in (dict(), dict(act=3), dict(p=0.5), dict(odd=(1, 1, 1))):
            asked, parts = _fits(*size, kind, **kw)
            assert asked == 4 * 256 * N * (K + 1) == sum(last - first for first, last in parts), (asked, parts)


def test_uses_refuses():
    ends = (ctypes.c_int64 * 8)()

    def call(dy_stride=14, out=ends, **kw):
        return pc._lib().pcsr_linear_uses(ctypes.byref(_linear(**kw)), P, dy_stride, out)

    assert call() == OK and call(dy_stride=13) == INVALID and call(out=None) == INVALID and call(rows=0) == INVALID and call(type=3) == UNSUPPORTED
    assert pc._lib().pcsr_linear_uses(None, P, 14, ends) == INVALID


def test_host_tensors_are_refused():
    from paper_2605_15695_amd.dropout import Dropout, dropout
    from paper_2605_15695_amd.linear import FeedForward, Linear, linear

    X = torch.zeros(3, 4)
    with pytest.raises(ValueError):
        dropout(X, 0.5, 1)
    with pytest.raises(ValueError):
        Dropout(0.5)(X)
    with pytest.raises(ValueError):
        linear(X, torch.zeros(5, 4))
    with pytest.raises(ValueError):
        Linear(4, 5)(X)
    with pytest.raises(ValueError):
        FeedForward(4, 5)(X)
    for p in (-0.5, 1.5, float("nan")):
        with pytest.raises(ValueError):
            Dropout(p)
        with pytest.raises(ValueError):
            Linear(4, 5, p=p)
    for seed in (1 << 64, -(1 << 63) - 1, 0.5):
        with pytest.raises(ValueError):
            Dropout(0.5, seed=seed)
    assert Dropout(0.5, seed=(1 << 64) - 1).counter.tolist() == [-1, 0]


def test_modules_keep_what_they_are_given():
    from paper_2605_15695_amd.dropout import Dropout
    from paper_2605_15695_amd.linear import FeedForward, Linear

    torch.manual_seed(1)
    a, b = Dropout(0.5), Dropout(0.5)
    torch.manual_seed(1)
    c = Dropout(0.5)
    assert a.counter.tolist() == c.counter.tolist() != b.counter.tolist()
    assert a(X := torch.ones(2, 2)) is X if not a.train(False).training else False
    assert set(Linear(3, 4).state_dict()) == {"weight", "bias"} and set(Linear(3, 4, False, p=0.1).state_dict()) == {"weight", "counter"}
    block = FeedForward(3, 8, "silu", 0.1)
    assert block.first.activation == "silu" and block.second.weight.shape == (3, 8)


def test_models_with_dropout_and_blocks_between_the_layers():
    from paper_2605_15695_amd.gnn import make_model

    def names(**kw):
        return [type(m).__name__ for m in make_model("gcn", None, 4, 8, 4, 3, **kw)]

    assert names() == ["GCNLayer", "ReLU"] * 2 + ["GCNLayer"]
    assert names(dropout=0.5) == ["GCNLayer", "ReLU", "Dropout"] * 2 + ["GCNLayer"]
    assert names(norm_groups=2, feed_forward=4) == ["GCNLayer", "GroupNorm", "FeedForward"] * 2 + ["GCNLayer"]
    model = make_model("gin", None, 4, 8, 4, 3, dropout=0.5, feed_forward=4)
    assert model[2].first.p == model[2].second.p == model[3].p == 0.5 and model[2].first.weight.shape == (32, 8)
    with pytest.raises(ValueError):
        make_model("gcn", None, 4, 8, 4, 3, dropout=1.5)
