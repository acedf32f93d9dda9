"""The gated delta rule over few steps (GPU): one after the other, or by pieces where there are few sequences, as the header says."""
import pytest
import torch

from test_gpu_learning import BACK, Delta, apex  # noqa: F401

pytestmark = pytest.mark.gpu
NAN = float("nan")


def some(c, sequences):
    """The same case, of these sequences alone."""
    d = object.__new__(Delta)
    d.__dict__.update(c.__dict__)
    S = len(range(*sequences.indices(c.sizes[0])))
    d.sizes = (S, *c.sizes[1:])
    for n in ("q", "k", "v", "do", "g", "beta", "h0", "dh_last", "discount", "length"):
        setattr(d, n, getattr(c, n)[sequences])
    return d


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [8, 9, 12, 16, 17])
def test_few_and_many_sequences_of_few_steps(apex, T, dtype):  # noqa: F811
    """150 sequences of 2 heads are by steps up to 16, one of them up to 8: both are within the same bounds, and to the bit the same where
    both go one way."""
    c = Delta(150, T, 1, 2, 40, 50, dtype, seed=T, cut=True, ragged=True)
    every = c.run(apex)
    c.check(every)
    for s in (0, 7):
        d = some(c, slice(s, s + 1))
        alone = d.run(apex)
        d.check(alone)
        if not 9 <= T <= 16:
            for n in ("o", "h_last") + BACK:
                assert torch.equal(alone[n], every[n][s:s + 1]), n


@pytest.mark.parametrize("S,T", [(1, 1), (1, 8), (150, 9), (150, 16)])
@pytest.mark.parametrize("bad", [NAN, float("inf")])
def test_steps_one_after_the_other_keep_out_what_has_ended(apex, S, T, bad):  # noqa: F811
    """In inputs and in the start state, behind an episode's end and behind a decay of 0."""
    c = Delta(S, T, 1, 2, 20, 30, "f32", seed=1)
    c.discount = torch.ones((S, T), device="cuda:0")
    end = min(2, T - 1)
    c.discount[:, end] = 0.0
    call = lambda: apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, h0=c.h0, discount=c.discount, scale=c.scale, carry=True)  # noqa: E731
    rc, clean = call()
    assert rc == apex.OK
    for n in ("q", "k", "v", "g", "beta", "h0"):
        held = getattr(c, n).clone()
        getattr(c, n)[:, 0] = bad
        rc, got = call()
        setattr(c, n, held)
        assert rc == apex.OK
        assert torch.equal(got["o"][:, end + 1:], clean["o"][:, end + 1:]) and torch.equal(got["h_last"], clean["h_last"]), n
    if T > 3:
        c.discount[:, end] = 1.0
        c.g[:, 3] = -float("inf")
        rc, clean = call()
        c.v[:, 1] = bad
        rc, got = call()
        assert rc == apex.OK and torch.equal(got["o"][:, 3:], clean["o"][:, 3:]) and torch.equal(got["h_last"], clean["h_last"])
        assert got["o"][:, 1].isnan().any() or got["o"][:, 1].isinf().any()
