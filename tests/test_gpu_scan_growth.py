"""Given factors above 1: products over many steps that leave the range of 32-bit numbers where the recurrence itself does not."""
import numpy as np
import pytest
import torch

import operators_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


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


def check(apex, g, x, dh, dtype, h0=None, dh_last=None, discount=None, length=None):
    S, T, D = g.shape
    dev = lambda a, t=torch.float32: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0").to(t)  # noqa: E731
    dt = DTYPES[dtype]
    g, x, dh, h0, dh_last = dev(g, dt), dev(x, dt), dev(dh, dt), dev(h0), dev(dh_last)
    k = dict(gate="given", discount=dev(discount), length=dev(length, torch.int32))
    want = plain.scan(plain.f64(g), plain.f64(x), "given", discount, length, plain.f64(h0), plain.f64(dh), plain.f64(dh_last))
    assert all(np.abs(want[n]).max() < 1e37 for n in ("h", "dg", "dx", "dh0"))
    got, again = [], []
    for out in (got, again):
        rc, forward = apex.gated_scan(g, x, h0=h0, carry=True, **k)
        assert rc == apex.OK
        rc, back = apex.gated_scan_backward(g, x, dh, forward["carry"], dh_last=dh_last, **k)
        assert rc == apex.OK
        out.append({**forward, **back})
    for n in ("h", "dg", "dx", "h_last", "dh0"):
        row_by_row(got[0][n], want[n], want[n + "_err"], dt if n in ("h", "dg", "dx") else torch.float32, n)
        assert torch.equal(got[0][n], again[0][n]), n


LENGTHS = [11, 12, 64, 100, 128, 129, 300, 700, 2500]


@pytest.mark.parametrize("T", LENGTHS)
@pytest.mark.parametrize("factor", [1.5, -3.0, 1e30, 3e38])
def test_nothing_grows_to_nothing(apex, T, factor):
    """No input, no start: every state is 0 whatever the factors, and so is every gradient of no gradient."""
    zero = np.zeros((2, T, 70), np.float32)
    check(apex, np.full((2, T, 70), factor, np.float32), zero, zero, "f32")
    check(apex, np.full((2, T, 70), factor, np.float32), zero, zero, "bf16", np.zeros((2, 70), np.float32), np.zeros((2, 70), np.float32))


@pytest.mark.parametrize("T", LENGTHS)
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("period", [3, 40, 150])
def test_factors_that_grow_and_then_shrink(apex, T, dtype, period):
    """Some powers of 2 up and down again, `period` steps each way at another beat in every channel, from small states."""
    rng = np.random.default_rng(T + period)
    S, D = 2, 131
    step = {3: 2.0 ** 30, 40: 2.0, 150: 2.0 ** 0.5}[period]
    beat = (np.arange(T)[:, None] + rng.integers(0, 2 * period, D)) // period % 2
    g = np.broadcast_to(np.where(beat == 0, step, 1 / step), (S, T, D)).astype(np.float32)
    small = 2.0 ** -75 if period == 150 else 2.0 ** -60
    x, dh = (rng.standard_normal((S, T, D)).astype(np.float32) * small for _ in range(2))
    h0, dh_last = (rng.standard_normal((S, D)).astype(np.float32) * small for _ in range(2))
    check(apex, g, x, dh, dtype, h0, dh_last)
    discount = np.where(rng.random((S, T)) < 0.01, 0.0, 0.9).astype(np.float32)
    check(apex, g, x, dh, dtype, h0, dh_last, discount, np.array([T, max(1, T - T // 3)], np.int32))


@pytest.mark.parametrize("T", LENGTHS)
@pytest.mark.parametrize("spread", [0.05, 0.5, 1.0])
def test_factors_around_one(apex, T, spread):
    """A walk of the products: stretches that grow beyond the bound beside others that do not."""
    rng = np.random.default_rng(T)
    S, D = 3, 200
    place, walk = np.zeros((S, D)), np.zeros((S, T, D))                # a walk that is drawn back to 0, and its steps
    for t in range(T):
        next_place = 0.98 * place + rng.standard_normal((S, D)) * spread
        walk[:, t], place = next_place - place, next_place
    g = (np.exp(walk) * rng.choice([-1, 1], (S, T, D))).astype(np.float32)
    x, dh = (rng.standard_normal((S, T, D)).astype(np.float32) * 1e-9 for _ in range(2))
    h0, dh_last = (rng.standard_normal((S, D)).astype(np.float32) * 1e-9 for _ in range(2))
    check(apex, g, x, dh, "f32", h0, dh_last, None, np.array([T, T // 2, max(0, T - 70)], np.int32))
    check(apex, g, x, dh, "bf16", h0, dh_last, np.where(rng.random((S, T)) < 0.02, 0.0, 1.0).astype(np.float32), None)


def test_one_large_factor(apex):
    """A single step far above 1 in one channel of one sequence, in every place of a stretch of tiles; strided inputs."""
    rng = np.random.default_rng(5)
    S, T, D = 1, 700, 140
    for at in (0, 5, 63, 64, 130, 200, 255, 256, 400, 511, 512, 699):
        g = rng.uniform(0.5, 1.0, (S, T, D)).astype(np.float32)
        g[0, at, 133] = 2.0 ** 40
        x, dh = (rng.standard_normal((S, T, D)).astype(np.float32) for _ in range(2))
        check(apex, g, x, dh, "f32", rng.standard_normal((S, D)).astype(np.float32), rng.standard_normal((S, D)).astype(np.float32))


def test_numbers_that_are_none(apex):
    """Where factors go from step to step: NaN and infinities pass to the steps behind them and no further than a cut."""
    S, T, D = 2, 400, 33
    g, x = np.full((S, T, D), 2.0, np.float32), np.zeros((S, T, D), np.float32)
    discount = np.ones((S, T), np.float32)
    discount[0, 200] = 0.0
    x[0, 100, 3], x[1, 300, 4] = np.nan, np.inf
    dev = lambda a: torch.from_numpy(a).to("cuda:0")  # noqa: E731
    rc, out = apex.gated_scan(dev(g), dev(x), gate="given", discount=dev(discount))
    assert rc == apex.OK
    want = np.zeros((S, T, D), np.float32)
    want[0, 100:201, 3], want[1, 300:, 4] = np.nan, np.inf
    assert np.array_equal(out["h"].cpu().numpy(), want, equal_nan=True)
    assert np.array_equal(out["h_last"].cpu().numpy(), want[:, -1])
