"""Distillation where the student is near its teacher or the named tokens have little of the mass: the loss is what the two halves of
its definition, which cancel, leave."""
import numpy as np
import pytest
import torch

import divergence_plain as near
import operators_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def row_by_row(got, want, err, dtype, what):
    got = plain.f64(got)
    bound = err + plain.rounding(want, dtype)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), "%s: %d of %d off, first at %s: %g for %g, bound %g" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], bound[bad][0])


def case(N, V, K, dtype, apart, tau, rest, spread=2.0, seed=0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.standard_normal((N, V)) * spread).astype(np.float32)).to(DTYPES[dtype])
    t = plain.f64(z) + rng.standard_normal((N, V)) * apart
    index = np.argsort(-t, axis=1)[:, :K].astype(np.int32)
    value = np.take_along_axis(t, index, 1).astype(np.float32)
    y = t / tau
    lse = (y.max(1) + np.log(np.exp(y - y.max(1, keepdims=True)).sum(1))).astype(np.float32) if rest else None
    weight = rng.uniform(0.1, 1.0, N).astype(np.float32)
    return z, index, value, lse, weight


def run(apex, z, index, value, lse, weight, tau):
    dev = lambda a: None if a is None else torch.as_tensor(a).to("cuda:0")  # noqa: E731
    rc, out = apex.distill_topk(dev(z), dev(index), dev(value), weight=dev(weight), top_lse=dev(lse), temperature=tau)
    assert rc == apex.OK
    torch.cuda.synchronize()
    want = near.distill(plain.f64(z), index, value.astype(np.float64), tau, None if lse is None else lse.astype(np.float64), weight)
    for n, dtype in (("loss", torch.float32), ("lse", torch.float32), ("grad", z.dtype)):
        row_by_row(out[n], want[n], want[n + "_err"], dtype, n)
    return plain.f64(out["loss"]), want


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,V,K,apart,tau", [(40, 40000, 1, 0.7, 4.0), (20, 40000, 16, 0.7, 4.0), (10, 100000, 1, 0.7, 4.0),
                                             (30, 20216, 13, 0.7, 1.5), (30, 3001, 2, 0.05, 2.0), (8, 200000, 3, 0.7, 4.0),
                                             (30, 1000, 40, 0.01, 0.25), (30, 513, 500, 0.02, 1.0), (300, 40000, 1, 0.7, 4.0)])
def test_losses_with_a_rest_class(apex, N, V, K, apart, tau, dtype):
    """Little mass named, as much, and nearly all of it."""
    loss, want = run(apex, *case(N, V, K, dtype, apart, tau, True, seed=V + K), tau)
    assert (loss > 0).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V", [2, 9, 64, 1000])
@pytest.mark.parametrize("apart", [0.5, 1e-2, 1e-3])
def test_losses_where_every_token_is_named(apex, V, apart, rest):
    run(apex, *case(25, V, V, "f32", apart, 1.0, rest, seed=V), 1.0)


@pytest.mark.parametrize("K", [1, 5, 64])
@pytest.mark.parametrize("tau", [1.0, 4.0])
def test_a_student_that_equals_its_teacher(apex, K, tau):
    """What the rounding of top_lse leaves of the loss, and no less than nothing."""
    loss, want = run(apex, *case(64, 40000, K, "f32", 0.0, tau, True, seed=K), tau)
    assert (loss >= 0).all() and (loss < 1e-10).all()


def test_the_rest_of_a_sharp_student_and_of_a_sharp_teacher(apex):
    """The student gives the tokens not named next to nothing, or the teacher does."""
    for student, teacher in ((12.0, 0.0), (0.0, 12.0), (5.0, 5.5), (30.0, 1.0)):
        z, index, _, _, weight = case(20, 3000, 4, "f32", 0.0, 1.0, True, seed=3)
        base = plain.f64(z)
        t = base.copy()
        np.put_along_axis(t, index.astype(np.int64), np.take_along_axis(base, index.astype(np.int64), 1) + teacher, 1)
        s = base.copy()
        np.put_along_axis(s, index.astype(np.int64), np.take_along_axis(base, index.astype(np.int64), 1) + student, 1)
        value = np.take_along_axis(t, index.astype(np.int64), 1).astype(np.float32)
        lse = (t.max(1) + np.log(np.exp(t - t.max(1, keepdims=True)).sum(1))).astype(np.float32)
        run(apex, torch.from_numpy(s.astype(np.float32)), index, value, lse, weight, 1.0)
