"""What the calls around the graph layers refuse, and what they ask for, without a GPU: the C entry points check their
arguments before they touch the device, and the Python ones before they call."""
import ctypes

import pytest

from paper_2605_15695_amd import binding as pc

torch = pytest.importorskip("torch")

OK, INVALID, UNSUPPORTED, TOO_LARGE = pc.PCSR_OK, pc.PCSR_E_INVALID_ARG, pc.PCSR_E_UNSUPPORTED, pc.PCSR_E_TOO_LARGE
P = 4096  # an address: nothing is read there


def test_embedding_entry_points():
    lib = pc._lib()

    def fwd(n=3, rows=5, d=4, type=0, ids=P, table=P, stride=4, out=P):
        return lib.pcsr_embed(n, rows, d, type, ids, 0, table, stride, 1.0, out, None)

    def bwd(n=3, rows=5, d=4, type=0, ids=P, dout=P, stride=4, grad=P, ws=P):
        return lib.pcsr_embed_backward(n, rows, d, type, ids, 0, dout, stride, 1.0, grad, ws, None)

    for call in (fwd, bwd):
        for bad in (dict(n=-1), dict(rows=-1), dict(d=0), dict(stride=3), dict(ids=None)):
            assert call(**bad) == INVALID, bad
        for bad in (dict(type=3), dict(type=-1)):
            assert call(**bad) == UNSUPPORTED
        for bad in (dict(n=1 << 31), dict(rows=1 << 31), dict(d=(1 << 23) + 1, stride=1 << 24), dict(stride=(1 << 31) + 1)):
            assert call(**bad) == TOO_LARGE, bad
    assert fwd(out=None) == INVALID and fwd(table=None) == INVALID and fwd(n=0, ids=None, out=None) == OK
    assert bwd(dout=None) == INVALID and bwd(grad=None) == INVALID and bwd(rows=0, grad=None) == OK
    assert lib.pcsr_embed_workspace(4096, 1000, 64) == 0  # few ids need none
    need = lib.pcsr_embed_workspace(100_000, 1000, 64)
    assert need > 100_000 * 16 and bwd(n=100_000, rows=1000, ws=None) == INVALID


def _norm(**kw):
    a = pc.pcsr_norm_t(10, 12, 3, 1, None, 0, 0, 0, 0, P, 12, None, None, 1e-5, P, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_norm_entry_points():
    lib = pc._lib()

    def fwd(y=P, ws=P, **kw):
        return lib.pcsr_norm(ctypes.byref(_norm(**kw)), y, ws, None)

    def bwd(dy=P, stride=12, dx=P, dw=P, db=P, ws=P, **kw):
        return lib.pcsr_norm_backward(ctypes.byref(_norm(**kw)), dy, stride, dx, dw, db, ws, None)

    for call in (fwd, bwd):
        for bad in (dict(rows=-1), dict(channels=0), dict(groups=5), dict(groups=0), dict(graphs=0), dict(graphs=3), dict(x_stride=11),
                    dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(mean=None), dict(rstd=None)):
            assert call(**bad) == INVALID, bad
        for bad in (dict(type=3), dict(param_type=-1), dict(act=4), dict(channels=2049, groups=1, x_stride=2049),
                    dict(type=1, channels=4097, groups=1, x_stride=4097)):
            assert call(**bad) == UNSUPPORTED, bad
        assert call(x_stride=(1 << 31) + 1) == TOO_LARGE
    assert fwd(y=None) == INVALID and fwd(rows=0, y=None) == OK
    many = dict(rows=1 << 25, graphs=1 << 25, channels=512, groups=1, x_stride=512, type=0)  # a workgroup each: more threads than a launch has
    assert fwd(**many) == TOO_LARGE
    assert bwd(dy=None) == INVALID and bwd(stride=11) == INVALID and bwd(dx=None, dw=None, db=None) == OK
    big = _norm(rows=100_000, channels=64, groups=4, x_stride=64)
    assert lib.pcsr_norm_workspace(ctypes.byref(big), 0) > 0
    assert lib.pcsr_norm(ctypes.byref(big), P, None, None) == INVALID
    assert lib.pcsr_norm(None, P, P, None) == INVALID and lib.pcsr_norm_workspace(None, 0) == 0


def test_orthogonalise_entry_point():
    lib = pc._lib()
    co = (ctypes.c_double * 48)(*([3.4445, -4.7750, 2.0315] * 16))

    def call(matrices=None, type=0, steps=5, coefficients=co, ws=P, **kw):
        how = pc.pcsr_ortho_t(type, steps, ctypes.addressof(coefficients) if coefficients is not None else None, 0, 0, 0.0, 0.0)
        m = pc.pcsr_matrix_t(P, None, P, 300, 200, 200, 0, 200, 0.0, 0)
        for k, v in kw.items():
            setattr(m, k, v)
        many = (pc.pcsr_matrix_t * 1)(m)
        return lib.pcsr_orthogonalize(many, 1, ctypes.byref(how), ws, None), lib.pcsr_ortho_workspace(many, 1, ctypes.byref(how))

    for bad in (dict(steps=0), dict(steps=17), dict(coefficients=None), dict(rows=-1), dict(grad=None), dict(out=None), dict(grad_ld=199),
                dict(out_ld=199), dict(buf=P, buf_ld=199)):
        assert call(**bad) == (INVALID, 0), bad
    assert call(type=3) == (UNSUPPORTED, 0)
    assert call(rows=(1 << 17) + 1)[0] == TOO_LARGE
    rc, need = call(ws=None)
    assert rc == INVALID and need > 300 * 200 * 4
    assert call(rows=100, cols=128, ws=None, grad_ld=128, out_ld=128, coefficients=None)[0] == INVALID
    grows = (ctypes.c_double * 48)(*([1e9, 0.0, 0.0] * 16))
    assert call(coefficients=grows)[0] == UNSUPPORTED
    assert call(rows=0) == (OK, 0)
    how = pc.pcsr_ortho_t(0, 5, ctypes.addressof(co), 0, 0, 0.0, 0.0)
    assert lib.pcsr_orthogonalize(None, 0, ctypes.byref(how), None, None) == OK


def test_host_tensors_are_refused():
    from paper_2605_15695_amd.embedding import NodeEmbedding, embedding
    from paper_2605_15695_amd.muon import Muon, orthogonalize
    from paper_2605_15695_amd.norm import GroupNorm, group_norm

    with pytest.raises(ValueError):
        embedding(torch.zeros(3, dtype=torch.int64), torch.zeros(4, 5))
    with pytest.raises(ValueError):
        NodeEmbedding(4, 5)(torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        group_norm(torch.zeros(3, 4), 2)
    with pytest.raises(ValueError):
        GroupNorm(2, 4)(torch.zeros(3, 4))
    with pytest.raises(ValueError):
        orthogonalize(torch.zeros(3, 4))
    p = torch.nn.Parameter(torch.zeros(3, 4))
    opt = Muon([p])
    opt.step()  # nothing has a gradient
    p.grad = torch.ones(3, 4)
    with pytest.raises(ValueError):
        opt.step()
    with pytest.raises(ValueError):
        opt.add_param_group({"params": [torch.nn.Parameter(torch.zeros(3))]})
    assert len(opt.param_groups) == 1


def test_models_with_norms_between_the_layers():
    from paper_2605_15695_amd.gnn import make_model
    from paper_2605_15695_amd.norm import GroupNorm

    plain, normed = (make_model("gin", None, 4, 8, 4, 3, norm_groups=g) for g in (0, 2))
    assert [type(m).__name__ for m in plain] == ["GINLayer", "ReLU"] * 2 + ["GINLayer"]
    assert [type(m).__name__ for m in normed] == ["GINLayer", "GroupNorm"] * 2 + ["GINLayer"]
    assert all(m.activation == "relu" and m.groups == 2 for m in normed if isinstance(m, GroupNorm))
    with pytest.raises(ValueError):
        plain(torch.zeros(3, 4), offsets=torch.zeros(2))
