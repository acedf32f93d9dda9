"""What the gated delta rule's products of two 32-bit numbers may be off by (GPU)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# Two parts of 8 bits cut off 1 + 2^-7 - 2^-23 leave 1, 255 * 2^-15 and 255 * 2^-23: the products of the second and third of them, which
# six products of parts leave out, are then as large as they can be, 2^-21 of the number's square.
X = 1 + 2.0 ** -7 - 2.0 ** -23
# Parts that are rounded leave out at most 2^-24; of the additions, those of the second part to the first's product are not exact, two of
# them, each off by 2^-23 at most (whether the matrix instruction rounds or cuts off).
LIMIT = 5 * 2.0 ** -24


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def numbers(S, seed):
    """X in different signs and powers of two, [S]."""
    g = torch.Generator().manual_seed(seed)
    sign = 1 - 2 * torch.randint(0, 2, (S,), generator=g)
    return (X * sign * 2.0 ** torch.randint(-20, 20, (S,), generator=g)).float().cuda()


def run(apex, T, q, k, v, beta, h0, do, dh_last):
    """One state of one number for each of S sequences; q, k, v and do [S,T]."""
    S = q.shape[0]
    wide = [x.view(S, T, 1, 1) for x in (q, k, v, do)]
    g = torch.zeros((S, T, 1), device="cuda:0")
    beta, h0, dh_last = beta.view(S, T, 1), h0.view(S, 1, 1, 1), dh_last.view(S, 1, 1, 1)
    rc, out = apex.delta_rule(*wide[:3], g, beta, h0=h0, carry=True)
    assert rc == apex.OK
    rc, back = apex.delta_rule_backward(*wide[:3], g, beta, wide[3], out["carry"], dh_last=dh_last)
    assert rc == apex.OK
    torch.cuda.synchronize()
    return {n: x.flatten(1).double() for n, x in {**out, **back}.items()}


def close(got, a, b, what):
    want = a.double() * b.double()
    off = ((got - want) / want).abs().max()
    assert off <= LIMIT, "%s: %.3g of the product, limit %.3g" % (what, off, LIMIT)


@pytest.mark.parametrize("T", [17, 150])
def test_products_of_32_bit_numbers_have_their_bits(apex, T):
    S = 40
    zeros, (a, b, c) = torch.zeros((S, T), device="cuda:0"), (numbers(S, i) for i in range(3))
    first = zeros.clone()
    first[:, 0] = 1.0
    # a state that stays: o = q h0, dq = do h0, dh0 = q do
    got = run(apex, T, first * a[:, None], zeros, zeros, zeros, b, first * c[:, None], torch.zeros(S, device="cuda:0"))
    close(got["o"][:, 0], a, b, "o from the state")
    close(got["dq"][:, 0], b, c, "dq from the state")
    close(got["dh0"][:, 0], a, c, "dh0")
    # one step that is kept: S = k v, o = q S behind it, dv = k dh_last, dk = v dh_last
    got = run(apex, T, torch.ones_like(zeros), first * a[:, None], first * b[:, None], first, torch.zeros(S, device="cuda:0"), zeros, c)
    close(got["o"][:, 16], a, b, "o from an earlier step")
    close(got["h_last"][:, 0], a, b, "h_last")
    close(got["dv"][:, 0], a, c, "dv")
    close(got["dk"][:, 0], b, c, "dk")
