"""The plain forms of the learning step's operators against differences, and what the library's entry points refuse (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import learning_plain as plain


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


@pytest.mark.parametrize("cut,ragged", [(False, False), (True, True)])
def test_gradient_of_the_delta_rule_against_differences(cut, ragged):
    rng = np.random.default_rng(3)
    S, T, Hk, H, Dk, Dv = 2, 7, 1, 2, 3, 2
    x = dict(q=rng.standard_normal((S, T, Hk, Dk)), k=rng.standard_normal((S, T, Hk, Dk)) * 0.6, v=rng.standard_normal((S, T, H, Dv)),
             g=-rng.random((S, T, H)), beta=rng.random((S, T, H)), h0=rng.standard_normal((S, H, Dk, Dv)))
    more = dict(scale=0.7, discount=np.where(rng.random((S, T)) < 0.3, 0.0, 1.0) if cut else None, length=np.array([T, 4]) if ragged else None)
    do, dh = rng.standard_normal((S, T, H, Dv)), rng.standard_normal((S, H, Dk, Dv))
    want = plain.delta(**x, **more, do=do, dh_last=dh)

    def value(**changed):
        r = plain.delta(**{**x, **changed}, **more)
        return (r["o"] * do).sum() + (r["h_last"] * dh).sum()
    for name in x:
        grad = want["d" + name]
        for at in np.ndindex(x[name].shape):
            d = np.zeros(x[name].shape)
            d[at] = 1e-5
            slope = (value(**{name: x[name] + d}) - value(**{name: x[name] - d})) / 2e-5
            assert abs(slope - grad[at]) < 1e-8 * (1 + abs(slope)), (name, at)


def test_gradient_of_the_embedding_against_differences():
    rng = np.random.default_rng(1)
    table, token, dout = rng.standard_normal((5, 3)), np.array([0, 4, 0, -1, 7, 2]), rng.standard_normal((6, 3))
    grad, _ = plain.embedding_backward(dout, token, 5, 1.5)
    for at in np.ndindex(table.shape):
        d = np.zeros(table.shape)
        d[at] = 1e-6
        slope = ((plain.embedding(table + d, token, 1.5) - plain.embedding(table - d, token, 1.5)) * dout).sum() / 2e-6
        assert abs(slope - grad[at]) < 1e-8


A = 1 << 20      # an address that nothing is launched with


def delta_args(**changed):
    x = dict(S=2, T=70, Hk=2, H=4, Dk=8, Dv=8, dtype=1, q=A, q_seq=70 * 16, q_time=16, k=A, k_seq=70 * 16, k_time=16, v=A, v_seq=70 * 32, v_time=32,
             g=A, beta=A, scale=1.0, discount=None, length=None)
    x.update(changed)
    return x


FORWARD = dict(h0=None, o=A, h_last=None, carry=None, workspace=A, stream=None)
BACKWARD = dict(carry=A, do=A, dh_last=None, dq=A, dq_seq=70 * 16, dq_time=16, dk=A, dk_seq=70 * 16, dk_time=16, dv=A, dv_seq=70 * 32, dv_time=32,
                dg=A, dbeta=A, dh0=None, workspace=A, stream=None)
NAN, INF = float("nan"), float("inf")
BAD = [dict(S=0), dict(T=0), dict(Hk=0), dict(H=0), dict(Dk=0), dict(Dv=0), dict(H=3), dict(dtype=3), dict(dtype=-1), dict(q=None), dict(k=None),
       dict(v=None), dict(g=None), dict(beta=None), dict(q=A + 1), dict(g=A + 2), dict(beta=A + 1), dict(discount=A + 2), dict(length=A + 1),
       dict(scale=NAN), dict(scale=INF), dict(workspace=None), dict(workspace=A + 128), dict(q_seq=1 << 63), dict(T=1 << 31)]
BAD_FORWARD = [dict(o=None), dict(o=A + 1), dict(h0=A + 2), dict(h_last=A + 2), dict(carry=A + 1)]
BAD_BACKWARD = [dict(carry=None), dict(do=None), dict(do=A + 1), dict(dq=None), dict(dk=None), dict(dv=None), dict(dg=None), dict(dbeta=None),
                dict(dq_time=15), dict(dk_seq=0), dict(dv_time=0), dict(dh_last=A + 1), dict(dh0=A + 1), dict(dq=A + 1), dict(dg=A + 3)]
LARGE = [dict(Dk=129), dict(Dv=129), dict(S=1 << 16, T=1 << 20)]


def given(apex, entry, groups, changed):
    x = {}
    for g in groups:
        x.update(g)
    assert set(changed) <= set(x)
    x.update(changed)
    return getattr(apex.lib, entry)(*x.values())


def test_delta_rule_refusals(apex):
    for entry, own, bad in (("apex_delta_rule", FORWARD, BAD_FORWARD), ("apex_delta_rule_backward", BACKWARD, BAD_BACKWARD)):
        for changed in BAD + bad:
            assert given(apex, entry, (delta_args(), own), changed) == apex.ERR_INVALID_ARG, (entry, changed)
        for changed in LARGE:
            assert given(apex, entry, (delta_args(), own), changed) == apex.ERR_TOO_LARGE, (entry, changed)


def test_delta_rule_workspace(apex):
    def need(*sizes):
        n = C.c_size_t(0)
        assert apex.lib.apex_delta_rule_workspace_bytes(*sizes, C.byref(n)) == apex.OK
        return n.value
    assert need(5, 1, 3, 8, 8, 0) == need(5, 8, 3, 8, 8, 0) == 0
    # what is enough for larger sizes is enough: also where those are computed step by step
    assert 0 < need(5, 16, 3, 8, 8, 0) <= need(500, 16, 3, 8, 8, 0) <= need(500, 17, 3, 8, 8, 0)
    assert 0 < need(1, 100, 3, 8, 8, 0) < need(2, 100, 3, 8, 8, 0) < need(2, 200, 3, 8, 8, 0)
    for sizes in ((2, 100, 3, 8, 8), (2, 1, 3, 128, 128)):
        assert need(*sizes, 1) > need(*sizes, 0)
    assert apex.lib.apex_delta_rule_workspace_bytes(1, 1, 1, 1, 1, 0, None) == apex.ERR_INVALID_ARG
    n = C.c_size_t(0)
    for sizes, rc in (((0, 1, 1, 1, 1), apex.ERR_INVALID_ARG), ((1, 1, 1, 129, 1), apex.ERR_TOO_LARGE), ((1 << 31, 1 << 30, 1 << 31, 1, 1), apex.ERR_TOO_LARGE)):
        assert apex.lib.apex_delta_rule_workspace_bytes(*sizes, 1, C.byref(n)) == rc


def test_embedding_refusals(apex):
    look = dict(N=3, V=9, D=4, dtype=0, table=A, table_stride=4, token=A, scale=1.0, out=A, out_stride=4, stream=None)
    back = dict(N=3, V=9, D=4, dtype=0, dout=A, dout_stride=4, token=A, scale=1.0, add=0, dtable=A, dtable_stride=4, workspace=A, stream=None)
    both = [dict(N=0), dict(V=0), dict(D=0), dict(dtype=5), dict(token=None), dict(token=A + 1), dict(scale=NAN), dict(scale=INF)]
    for entry, x, bad in (("apex_embedding", look, [dict(table=None), dict(out=None), dict(table=A + 2), dict(out=A + 1), dict(out_stride=3), dict(table_stride=1 << 62)]),
                          ("apex_embedding_backward", back, [dict(dout=None), dict(dtable=None), dict(workspace=None), dict(workspace=A + 4), dict(dtable_stride=3),
                                                             dict(dout=A + 2)])):
        for changed in both + bad:
            assert given(apex, entry, (x,), changed) == apex.ERR_INVALID_ARG, (entry, changed)
        for changed in (dict(N=apex.MAX_TOKENS + 1), dict(V=apex.MAX_VOCABULARY + 1), dict(D=apex.MAX_WIDTH + 1)):
            assert given(apex, entry, (x,), changed) == apex.ERR_TOO_LARGE, (entry, changed)
    n = C.c_size_t(0)
    assert apex.lib.apex_embedding_backward_workspace_bytes(1, 1, 1, None) == apex.ERR_INVALID_ARG
    assert apex.lib.apex_embedding_backward_workspace_bytes(0, 1, 1, C.byref(n)) == apex.ERR_INVALID_ARG
    assert apex.lib.apex_embedding_backward_workspace_bytes(1, 1, 1, C.byref(n)) == apex.OK and n.value > 0


def test_clipping_refusals(apex):
    def call(count=2, grad=(A, A), out=None, elements=(5, 6), dtype=(0, 1), max_norm=1.0, norm=None, workspace=A):
        array = lambda t, x: None if x is None else (t * max(len(x), 1))(*x)  # noqa: E731
        return apex.lib.apex_clip_gradients(count, array(C.c_void_p, grad), array(C.c_void_p, out), array(C.c_uint64, elements), array(C.c_int, dtype),
                                            max_norm, norm, workspace, None)
    for changed in (dict(grad=None), dict(elements=None), dict(dtype=None), dict(dtype=(0, 3)), dict(grad=(A, None)), dict(grad=(A + 1, A)), dict(grad=(A, A + 1)),
                    dict(out=(A, None)), dict(out=(A + 2, A)), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=NAN), dict(norm=A + 2), dict(workspace=None),
                    dict(workspace=A + 8)):
        assert call(**changed) == apex.ERR_INVALID_ARG, changed
    assert call(elements=((1 << 48) + 1, 1)) == apex.ERR_TOO_LARGE
    n = C.c_size_t(0)
    assert apex.lib.apex_clip_gradients_workspace_bytes(1, None) == apex.ERR_INVALID_ARG
    assert apex.lib.apex_clip_gradients_workspace_bytes(apex.MAX_TENSORS + 1, C.byref(n)) == apex.ERR_TOO_LARGE
    assert apex.lib.apex_clip_gradients_workspace_bytes(0, C.byref(n)) == apex.OK and n.value > 0


def test_what_the_calls_refuse_before_they_need_a_gpu(apex):
    import torch
    x = torch.zeros((1, 2, 1, 3))
    with pytest.raises(ValueError, match="carry"):
        apex.delta_rule(x, x, x, x, x, carry=True, out=dict(o=None), workspace=x)
    with pytest.raises(ValueError, match="add"):
        apex.embedding_backward(x, x, 3, add=True)
    with pytest.raises(ValueError, match="rows"):
        apex.embedding_backward(x, x, 3, out=dict(dtable=torch.zeros((4, 1))), workspace=x)
    with pytest.raises(ValueError, match="laid out"):
        apex.clip_gradients([torch.zeros((2, 3))], 1.0, out=[torch.zeros((3, 2)).t()], norm=x, workspace=x)
    for call in (lambda: apex.embedding(torch.zeros((4, 3)), torch.zeros(2, dtype=torch.int32)),
                 lambda: apex.clip_gradients([torch.zeros(3)], 1.0, norm=x, workspace=x),
                 lambda: apex.delta_rule(x, x, x, x, x, out=dict(o=x), workspace=x)):
        with pytest.raises(AssertionError, match="device"):
            call()
