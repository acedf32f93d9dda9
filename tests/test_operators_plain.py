"""The operators' plain forms against differences, sums and frequencies, and the entry points' refusals (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import operators_plain as plain


# ------------------------------------------------------------------------------------------------ the plain forms themselves

@pytest.mark.parametrize("gate", ["given", "sigmoid"])
@pytest.mark.parametrize("cut", [False, True])
def test_scan_gradient_against_differences(gate, cut):
    """d(sum(dh h) + sum(dh_last h_last)) by central differences: step 1e-5, an error of the order of 1e-10."""
    rng = np.random.default_rng(3)
    S, T, D = 2, 9, 3
    g, x, h0 = rng.standard_normal((S, T, D)), rng.standard_normal((S, T, D)), rng.standard_normal((S, D))
    dh, dh_last = rng.standard_normal((S, T, D)), rng.standard_normal((S, D))
    discount = (rng.random((S, T)) > 0.3).astype(float) if cut else None
    length = np.array([9, 5]) if cut else None
    got = plain.scan(g, x, gate, discount, length, h0, dh, dh_last)

    def total(g, x, h0):
        o = plain.scan(g, x, gate, discount, length, h0)
        return (o["h"] * dh).sum() + (o["h_last"] * dh_last).sum()

    arrays = dict(dg=g, dx=x, dh0=h0)
    for name, a in arrays.items():
        for i in np.ndindex(a.shape):
            kept = a[i]
            a[i] = kept + 1e-5
            up = total(g, x, h0)
            a[i] = kept - 1e-5
            down = total(g, x, h0)
            a[i] = kept
            assert abs((up - down) / 2e-5 - got[name][i]) < 1e-8, (name, i)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distill_gradient_against_differences(rest, tau):
    rng = np.random.default_rng(4)
    N, V, K = 3, 11, 4
    z, t = rng.standard_normal((N, V)), rng.standard_normal((N, V))
    index = np.stack([rng.permutation(V)[:K] for _ in range(N)])
    index[1, 2], index[2, 1], index[2, 3] = -1, index[2, 0], V       # empty, named twice, out of range
    value = np.take_along_axis(t, np.clip(index, 0, V - 1), 1)
    top_lse = np.log(np.exp(t / tau).sum(1)) if rest else None
    weight = np.array([1.0, 0.5, 2.0])
    got = plain.distill(z, index, value, tau, top_lse, weight)
    assert (got["loss"] > 0).all()
    for i in np.ndindex(z.shape):
        kept = z[i]
        z[i] = kept + 1e-5
        up = plain.distill(z, index, value, tau, top_lse)["loss"]
        z[i] = kept - 1e-5
        down = plain.distill(z, index, value, tau, top_lse)["loss"]
        z[i] = kept
        assert abs((weight * (up - down)).sum() / 2e-5 - got["grad"][i]) < 1e-8, i
    assert np.allclose(got["grad"].sum(1), 0, atol=1e-12)            # a shift of all logits changes nothing


def test_distill_against_the_whole_distribution():
    """With every token named the loss is the divergence of the two softmaxes, with or without the rest class."""
    rng = np.random.default_rng(5)
    z, t = rng.standard_normal((2, 7)), rng.standard_normal((2, 7))
    index = np.stack([rng.permutation(7) for _ in range(2)])
    value = np.take_along_axis(t, index, 1)
    p, q = (np.exp(a) / np.exp(a).sum(1, keepdims=True) for a in (z, t))
    want = (q * np.log(q / p)).sum(1)
    assert np.allclose(plain.distill(z, index, value)["loss"], want, atol=1e-12)
    assert np.allclose(plain.distill(z, index, value, top_lse=np.log(np.exp(t).sum(1)))["loss"], want, atol=1e-12)


def test_verified_tokens_are_distributed_as_the_target():
    """The first token out, over 40,000 sequences that draft from q: frequencies of p within five standard deviations."""
    rng = np.random.default_rng(6)
    B, V = 40_000, 6
    q, p = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    token = rng.choice(V, size=(B, 1), p=q).astype(np.int32)
    rnd = rng.integers(0, 1 << 64, (B, 2), dtype=np.uint64)
    accepted, out = plain.verify(np.broadcast_to(p, (B, 2, V)), np.broadcast_to(q, (B, 1, V)), token, rnd)
    seen = np.bincount(out[:, 0], minlength=V) / B
    assert (np.abs(seen - p) < 5 * np.sqrt(p * (1 - p) / B)).all(), (seen, p)
    assert abs(accepted.mean() - np.minimum(p, q).sum()) < 5 * 0.5 / np.sqrt(B)


# --------------------------------------------------------------------------------------------------------------- refusals

@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


A = 1 << 20    # an address that no refused call looks behind


def scan_args(**k):
    d = dict(S=2, T=3, D=4, dtype=0, gate=1, g=A, gs=12, gt=4, x=A, xs=12, xt=4, discount=None, length=None, h0=None, h=A,
             h_last=None, carry=None, workspace=None, stream=None)
    assert set(k) <= set(d)
    return list({**d, **k}.values())


def back_args(**k):
    d = dict(S=2, T=3, D=4, dtype=0, gate=1, g=A, gs=12, gt=4, x=A, xs=12, xt=4, discount=None, length=None, carry=A, dh=A,
             dh_last=None, dg=A, dgs=12, dgt=4, dx=A, dxs=12, dxt=4, dh0=None, workspace=None, stream=None)
    assert set(k) <= set(d)
    return list({**d, **k}.values())


BIG = (1 << 64) - 1


@pytest.mark.parametrize("bad", [dict(S=0), dict(T=0), dict(D=0), dict(dtype=3), dict(dtype=-1), dict(gate=2), dict(gate=-1), dict(g=None),
                                 dict(x=None), dict(g=A + 2), dict(x=A + 1, dtype=1), dict(gs=BIG), dict(xt=BIG), dict(T=1 << 31),
                                 dict(discount=A + 2), dict(length=A + 1)])
def test_scan_refusals(apex, bad):
    assert apex.lib.apex_gated_scan(*scan_args(**bad)) == apex.ERR_INVALID_ARG
    assert apex.lib.apex_gated_scan_backward(*back_args(**bad)) == apex.ERR_INVALID_ARG


def test_scan_refusals_of_one_direction(apex):
    for bad in (dict(h=None), dict(h=A + 2), dict(h0=A + 1), dict(h_last=A + 2), dict(carry=A + 3)):
        assert apex.lib.apex_gated_scan(*scan_args(**bad)) == apex.ERR_INVALID_ARG, bad
    # gradients whose rows overlap: broadcast over sequences, over steps, interleaved too closely
    for bad in (dict(carry=None), dict(dh=None), dict(dg=None), dict(dx=None), dict(dg=A + 2), dict(dh0=A + 2), dict(dh_last=A + 1),
                dict(dgs=0), dict(dxs=0), dict(dgt=0), dict(dxt=3), dict(dgs=11), dict(dgs=4, dgt=4)):
        assert apex.lib.apex_gated_scan_backward(*back_args(**bad)) == apex.ERR_INVALID_ARG, bad
    for f, args in ((apex.lib.apex_gated_scan, scan_args), (apex.lib.apex_gated_scan_backward, back_args)):
        d = dict(gs=4, xs=4) if f is apex.lib.apex_gated_scan else dict(gs=4, xs=4, dgs=4, dgt=4 << 31, dxs=4, dxt=4 << 31)
        assert f(*args(S=1 << 31, D=4, **d)) == apex.ERR_TOO_LARGE


def test_distill_refusals(apex):
    def call(**k):
        d = dict(N=3, V=10, K=2, dtype=1, logits=A, stride=10, index=A, value_dtype=0, value=A, top_lse=None, weight=None, tau=1.0,
                 loss=A, lse=None, grad=A, grad_stride=10, workspace=None, stream=None)
        assert set(k) <= set(d)
        return apex.lib.apex_distill_topk(*{**d, **k}.values())
    for bad in (dict(N=0), dict(V=0), dict(K=0), dict(dtype=4), dict(value_dtype=-1), dict(logits=None), dict(index=None), dict(value=None),
                dict(loss=None), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")), dict(logits=A + 1),
                dict(stride=BIG), dict(grad=A + 1), dict(grad_stride=9), dict(grad_stride=BIG), dict(index=A + 2), dict(value=A + 2),
                dict(top_lse=A + 1), dict(weight=A + 2), dict(loss=A + 2), dict(lse=A + 2)):
        assert call(**bad) == apex.ERR_INVALID_ARG, bad
    assert call(V=apex.MAX_VOCABULARY + 1, stride=1 << 21, grad_stride=1 << 21) == apex.ERR_TOO_LARGE
    assert call(K=apex.MAX_TOP + 1) == apex.ERR_TOO_LARGE
    assert call(N=1 << 30) == apex.ERR_TOO_LARGE


def test_verify_refusals(apex):
    def call(**k):
        d = dict(B=2, G=3, V=10, dtype=0, target=A, ts=40, tr=10, draft=A, ds=30, dr=10, token=A, rnd=A, length=None, accepted=A,
                 token_out=A, workspace=A, stream=None)
        assert set(k) <= set(d)
        return apex.lib.apex_verify_draft(*{**d, **k}.values())
    for bad in (dict(B=0), dict(V=0), dict(dtype=3), dict(target=None), dict(draft=None), dict(token=None), dict(rnd=None),
                dict(accepted=None), dict(token_out=None), dict(workspace=None), dict(workspace=A + 128), dict(target=A + 2),
                dict(draft=A + 2), dict(ts=BIG), dict(dr=BIG), dict(token=A + 2), dict(rnd=A + 4), dict(length=A + 1),
                dict(accepted=A + 2), dict(token_out=A + 1)):
        assert call(**bad) == apex.ERR_INVALID_ARG, bad
    assert call(V=apex.MAX_VOCABULARY + 1) == apex.ERR_TOO_LARGE
    assert call(G=apex.MAX_DRAFT + 1) == apex.ERR_TOO_LARGE
    assert call(B=1 << 30) == apex.ERR_TOO_LARGE


def test_workspace_sizes(apex):
    lib, n = apex.lib, C.c_size_t(0)
    for f, sizes in ((lib.apex_gated_scan_workspace_bytes, (2, 3, 4)), (lib.apex_distill_topk_workspace_bytes, (2, 3)),
                     (lib.apex_verify_draft_workspace_bytes, (2, 3))):
        assert f(*sizes, C.byref(n)) == apex.OK
        assert f(*sizes, None) == apex.ERR_INVALID_ARG
        for i in range(len(sizes)):
            assert f(*(0 if j == i else s for j, s in enumerate(sizes)), C.byref(n)) == apex.ERR_INVALID_ARG
    for f in (lib.apex_distill_topk_workspace_bytes, lib.apex_verify_draft_workspace_bytes):
        assert f(1, apex.MAX_VOCABULARY, C.byref(n)) == apex.OK
        assert f(1, apex.MAX_VOCABULARY + 1, C.byref(n)) == apex.ERR_TOO_LARGE


def test_limits_match_the_header(apex):
    import os
    from conftest import ROOT
    text = open(os.path.join(ROOT, "include", "apex_replay.h")).read()
    for name, value in (("SCAN_CHUNK", apex.SCAN_CHUNK), ("MAX_VOCABULARY", apex.MAX_VOCABULARY), ("MAX_TOP", apex.MAX_TOP),
                        ("MAX_DRAFT", apex.MAX_DRAFT)):
        assert "#define APEX_%s %du" % (name, value) in text
    for name, value in (("F32", apex.F32), ("BF16", apex.BF16), ("F16", apex.F16), ("GATE_GIVEN", apex.GATES["given"]),
                        ("GATE_SIGMOID", apex.GATES["sigmoid"])):
        assert "APEX_%s = %d" % (name, value) in text


def test_binding_refuses_tensors_that_do_not_fit(apex):
    """Tensors of the CPU, and what is no tensor."""
    import torch

    class stream:
        cuda_stream = 0

    x = torch.zeros(2, 3, 4)
    with pytest.raises(AssertionError):
        apex._call.gated_scan(x, x, 1, None, None, None, x, None, None, None, stream)
    with pytest.raises(AssertionError):
        apex._call.gated_scan(None, None, 1, None, None, None, None, None, None, None, stream)
    with pytest.raises(TypeError):
        apex._call.gated_scan("g", None, 1, None, None, None, None, None, None, None, stream)
    with pytest.raises(AssertionError):
        apex._call.distill_topk(x[0], None, None, None, None, 1.0, None, None, None, None, stream)
    with pytest.raises(AssertionError):
        apex._call.verify_draft(None, None, None, None, None, None, None, None, stream)
