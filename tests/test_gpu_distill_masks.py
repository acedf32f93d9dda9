"""Distillation of logits far from 0: masks of the type's lowest value or of some large negative number, over the tokens that are not
named, over some of the row, over all of it; and large positive logits.  Only differences of logits matter, so that the
wanted values are those of the row less its largest logit, in 80 bits."""
import numpy as np
import pytest
import torch

import divergence_plain as near
import operators_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = [(3, 9, 4), (3, 700, 4), (300, 20001, 3), (3, 33001, 17), (2, 140001, 5), (300, 33003, 5)]   # all kinds of launches
LOOKED_AT = 4    # rows, the first ones


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def check(apex, z, index, value, lse, tau, in_place=False):
    dev = lambda a: None if a is None else torch.as_tensor(a).to("cuda:0")  # noqa: E731
    N, V = z.shape
    logits = dev(z)
    out = dict(loss=torch.empty(N, device="cuda:0"), lse=torch.empty(N, device="cuda:0"),
               grad=logits if in_place else torch.empty_like(logits))
    assert apex.distill_topk(logits, dev(index), dev(value), top_lse=dev(lse), temperature=tau, out=out)[0] == apex.OK
    torch.cuda.synchronize()
    out = {n: t[:LOOKED_AT] for n, t in out.items()}
    z, index, value, lse = plain.f64(z[:LOOKED_AT]), index[:LOOKED_AT], value[:LOOKED_AT], None if lse is None else lse[:LOOKED_AT]
    top = z.max(1, keepdims=True)
    want = near.distill(z - top, index, value.astype(np.float64), tau, None if lse is None else lse.astype(np.float64))
    with np.errstate(over="ignore"):
        wanted = {"loss": want["loss"].astype(np.float32).astype(np.float64), "grad": want["grad"],
                  "lse": (want["lse"] + top[:, 0] / tau).astype(np.float32).astype(np.float64)}
    err = {"loss": want["loss_err"], "grad": want["grad_err"], "lse": want["lse_err"] + near.U * np.abs(top[:, 0] / tau)}
    for n in ("loss", "lse", "grad"):
        got = plain.f64(out[n])
        dtype = DTYPES["f32"] if n != "grad" else logits.dtype
        same = (got == wanted[n]) & np.isinf(got)
        with np.errstate(invalid="ignore"):
            bad = ~(np.abs(got - wanted[n]) <= err[n] + plain.rounding(wanted[n], dtype)) & ~same
        assert not bad.any(), "%s: %d of %d off, first at %s: %g for %g, bound %g" % (
            n, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], wanted[n][bad][0], np.broadcast_to(err[n], got.shape)[bad][0])


def case(N, V, K, dtype, seed):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.standard_normal((N, V)).astype(np.float32) * 2).to(DTYPES[dtype])
    index = np.stack([rng.permutation(V)[:K] for _ in range(N)]).astype(np.int32)
    value = rng.standard_normal((N, K)).astype(np.float32)
    return rng, z, index, value


def masks(dtype):
    lowest = torch.finfo(DTYPES[dtype]).min
    return [lowest] + ([] if dtype == "f16" else [-1e9, -1e10, -3e38, -1.2e9])


@pytest.mark.parametrize("tau", [1.0, 0.25, 3.0])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,V,K", SIZES)
def test_masked_tokens_and_masked_rows(apex, N, V, K, dtype, tau):
    for i, low in enumerate(masks(dtype)):
        rng, z, index, value = case(N, V, K, dtype, V + i)
        z[0, torch.from_numpy(rng.random(V) < 0.7)] = low             # some of a row
        z[1] = low                                                    # all of it: every token is as likely as another
        check(apex, z, index, value, None, tau)
        if i == 0:
            check(apex, z, index, value, None, tau, in_place=True)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,V,K", SIZES)
def test_masks_over_all_that_is_not_named(apex, N, V, K, dtype):
    """A teacher that gives (nearly) all to the tokens it names, so that the loss is a number."""
    for i, low in enumerate(masks(dtype)):
        rng, z, index, value = case(N, V, K, dtype, V + i)
        keep = torch.from_numpy(index.astype(np.int64))
        masked = torch.full_like(z, low)
        masked.scatter_(1, keep, z.gather(1, keep))
        check(apex, masked, index, value, None, 1.0)
        lse = np.log(np.exp(value.astype(np.float64)).sum(1)).astype(np.float32)
        below = np.nextafter(lse, np.float32(-np.inf), dtype=np.float32)     # the teacher's sum is rounded down: no rest is left
        if low > -1e5:                                                # (f16) the rest has a probability that 64 bits do not hold
            continue
        check(apex, masked, index, value, below, 1.0)
        # every row of equal logits: the rest has its share
        lse = np.log(np.exp(value.astype(np.float64)).sum(1) + 1.0).astype(np.float32)
        check(apex, torch.full_like(z, low), index, value, lse, 1.0)


@pytest.mark.parametrize("N,V,K", SIZES)
def test_large_logits(apex, N, V, K):
    """Rows around large numbers, where neighbours in 32 bits are some way apart, and rows that hold the largest."""
    for i, (centre, apart) in enumerate(((1e6, 1.0), (1e7, 4.0), (3e8, 64.0), (7.5e8, 64.0), (1.6e9, 128.0), (3e9, 256.0), (1e12, 1e5))):
        for sign in (1, -1):
            rng, z, index, value = case(N, V, K, "f32", V + i)
            z = torch.from_numpy((sign * centre + np.round(rng.standard_normal((N, V))) * apart).astype(np.float32))
            check(apex, z, index, value, None, 1.0)
            check(apex, z, index, value, None, 50.0)
    rng, z, index, value = case(N, V, K, "f32", V)
    z[0, V // 2] = 3.4e38
    z[1, index[1, 0]] = 3e38
    check(apex, z, index, value, None, 1.0)


def test_students_and_teachers_of_any_temperature(apex):
    for tau in (1e-30, 1e-6, 1e-3, 1e3, 1e6, 1e30):
        _, z, index, value = case(4, 5000, 6, "f32", 3)
        index[:, 0] = plain.f64(z).argmax(1)
        for i in range(4):
            while len(set(index[i])) < 6:
                index[i, 1:] = np.random.default_rng(i).permutation(5000)[:5]
        value[:, 0] = 10.0
        check(apex, z, index, value, None, float(np.float32(tau)))
