"""What only large calls reach: outputs that are stored past the caches (above 32 MiB), more columns of channels than there are
ticket counters, chains longer than a tile looks back at once.  All of a large call's outputs equal those of the same call in parts
that are small enough, bit for bit, and some of them are compared with the plain forms."""
import numpy as np
import pytest
import torch

import operators_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PAST_CACHES = 32 << 20


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


def generator(seed):
    g = torch.Generator("cuda:0")
    g.manual_seed(seed)
    return g


# ----------------------------------------------------------------------------------------------------------- distill

@pytest.mark.parametrize("dtype,N,V,pad,K,part", [
    ("bf16", 700, 32768, 0, 20, 350), ("f16", 700, 32768, 7, 5, 350), ("bf16", 300, 65536, 0, 64, None), ("f16", 350, 65536 + 33, 1, 9, 200),
    ("f32", 120, 100003, 0, 3, 70), ("f32", 100, 131072, 0, 30, 60), ("bf16", 160, 131072, 0, 128, 100), ("bf16", 100, 200001, 0, 17, 70),
    ("f32", 9000, 1000, 0, 4, 8000)])
@pytest.mark.parametrize("rest", [False, True])
def test_gradients_past_the_caches(apex, dtype, N, V, pad, K, part, rest):
    g, dt = generator(V + K), DTYPES[dtype]
    assert N * V * dt.itemsize > PAST_CACHES
    held = torch.full((N, V + pad), float("nan"), dtype=dt, device="cuda:0")
    held[:, :V] = torch.randn((N, V), generator=g, device="cuda:0") * 2
    logits = held[:, :V]
    value, index = (logits.float() + torch.randn((N, V), generator=g, device="cuda:0") * 0.5).topk(K, 1)
    index = index.int()
    lse = torch.logsumexp(logits.float(), 1) + 0.3 if rest else None
    weight = torch.rand(N, generator=g, device="cuda:0") + 0.1
    rc, whole = apex.distill_topk(logits, index, value, weight=weight, top_lse=lse)
    assert rc == apex.OK
    for i in range(0, N, part or N):
        if part:      # (none where no part is small enough and goes by workgroups of the same size, sums in the same order)
            assert part * V * dt.itemsize <= PAST_CACHES
            at = slice(i, i + part)
            rc, out = apex.distill_topk(logits[at], index[at], value[at], weight=weight[at], top_lse=None if lse is None else lse[at])
            assert rc == apex.OK
            for n in ("loss", "lse", "grad"):
                assert torch.equal(out[n], whole[n][at]), n
    rows = [0, 1, N // 2, N - 2, N - 1]
    want = plain.distill(plain.f64(logits[rows]), index[rows].cpu().numpy(), plain.f64(value[rows]), 1.0,
                         None if lse is None else plain.f64(lse[rows]), plain.f64(weight[rows]))
    for n in ("loss", "lse", "grad"):
        row_by_row(whole[n][rows], want[n], want[n + "_err"], dt if n == "grad" else torch.float32, n)
    # in place, beside padding that stays as it is
    rc, out = apex.distill_topk(logits, index, value, weight=weight, top_lse=lse, out=dict(loss=torch.empty(N, device="cuda:0"), grad=logits))
    assert rc == apex.OK
    assert torch.equal(logits, whole["grad"]) and torch.equal(out["loss"], whole["loss"])
    assert torch.isnan(held[:, V:]).all()


# -------------------------------------------------------------------------------------------------------------- scan

class Scan:
    def __init__(self, S, T, D, dtype, gate, seed, cut, ragged):
        g, self.dtype, self.gate = generator(seed), DTYPES[dtype], gate
        rand = lambda *s: torch.randn(s, generator=g, device="cuda:0")  # noqa: E731
        self.g = ((rand(S, T, D) * 1.5 + 2) if gate == "sigmoid" else 1 - 0.4 * torch.rand((S, T, D), generator=g, device="cuda:0")).to(self.dtype)
        self.x, self.dh = rand(S, T, D).to(self.dtype), rand(S, T, D).to(self.dtype)
        self.h0, self.dh_last = rand(S, D), rand(S, D)
        self.discount = (torch.rand((S, T), generator=g, device="cuda:0") > 0.01).float() if cut else None
        self.length = torch.randint(0, T + 1, (S,), generator=g, device="cuda:0", dtype=torch.int32) if ragged else None
        if ragged:
            self.length[0] = T

    def run(self, apex, s=slice(None), d=slice(None), workspace=None):
        part = lambda a, *i: None if a is None else a[i].contiguous()  # noqa: E731
        every = slice(None)
        g, x, dh = (part(a, s, every, d) for a in (self.g, self.x, self.dh))
        k = dict(gate=self.gate, discount=part(self.discount, s), length=part(self.length, s), workspace=workspace)
        rc, out = apex.gated_scan(g, x, h0=part(self.h0, s, d), carry=True, **k)
        assert rc == apex.OK
        rc, back = apex.gated_scan_backward(g, x, dh, out["carry"], dh_last=part(self.dh_last, s, d), **k)
        assert rc == apex.OK
        return {**{n: out[n] for n in ("h", "h_last")}, **back}

    def check(self, got, s, d):
        """Against the plain form, for some sequences and channels."""
        host = lambda a: None if a is None else plain.f64(a[s])  # noqa: E731
        length = None if self.length is None else self.length[s].cpu().numpy()
        want = plain.scan(host(self.g)[:, :, d], host(self.x)[:, :, d], self.gate, host(self.discount), length, host(self.h0)[:, d],
                          host(self.dh)[:, :, d], host(self.dh_last)[:, d])
        for n in ("h", "dg", "dx", "h_last", "dh0"):
            row_by_row(got[n][s][..., d], want[n], want[n + "_err"], self.dtype if n in ("h", "dg", "dx") else torch.float32, n)


@pytest.mark.parametrize("S,T,D,dtype,gate,cut,ragged", [
    (2, 5000, 1003, "f32", "given", True, False), (2, 5000, 1003, "f32", "sigmoid", False, True), (1, 9000, 2048, "bf16", "sigmoid", False, False),
    (40, 100, 5000, "bf16", "sigmoid", True, True), (70, 128, 2000, "f16", "given", False, True), (600, 12, 2500, "bf16", "sigmoid", True, False)])
def test_states_and_gradients_past_the_caches(apex, S, T, D, dtype, gate, cut, ragged):
    c = Scan(S, T, D, dtype, gate, S + T, cut, ragged)
    assert S * T * D * c.dtype.itemsize > PAST_CACHES
    got = c.run(apex)
    part = 128 * max(1, (PAST_CACHES - 1) // (S * T * 128 * c.dtype.itemsize))
    assert part < D
    for i in range(0, D, part):
        few = c.run(apex, d=slice(i, i + part))
        for n in got:
            assert torch.equal(few[n], got[n][..., i:i + part]), n
    some = sorted({0, S // 2, S - 1})
    c.check(got, some, [0, 1, 127, 128, D // 2, D - 2, D - 1])


@pytest.mark.parametrize("S,T,D,dtype,gate", [(300, 150, 520, "bf16", "sigmoid"), (1100, 200, 100, "f32", "given"), (2, 130, 70000, "f16", "sigmoid")])
def test_more_columns_than_ticket_counters(apex, S, T, D, dtype, gate):
    """Columns of channels beyond 1024, and no multiple of it; one workspace in turn with calls of other shapes."""
    c, other = Scan(S, T, D, dtype, gate, S, True, True), Scan(3, 700, 300, "bf16", "sigmoid", 5, True, True)
    columns = S * -(-D // 128)
    assert columns > 1024 and columns % 1024
    space = max((apex.gated_scan_workspace(*a.g.shape) for a in (c, other)), key=lambda w: w.numel())
    got, beside = c.run(apex, workspace=space), other.run(apex, workspace=space)
    for _ in range(4):
        again, beside_again = c.run(apex, workspace=space), other.run(apex, workspace=space)
        for n in got:
            assert torch.equal(again[n], got[n]) and torch.equal(beside_again[n], beside[n]), n
    half = slice(0, S // 3) if S > 2 else slice(None)
    channels = slice(None) if S > 2 else slice(0, 12800)
    few = c.run(apex, s=half, d=channels)
    for n in got:
        assert torch.equal(few[n], got[n][half][..., channels]), n
    c.check(got, sorted({0, S // 2, S - 1}), [0, 1, D // 2, D - 1])
    other.check(beside, [0, 1, 2], [0, 299])


@pytest.mark.parametrize("dtype,gate,cut", [("f32", "sigmoid", False), ("bf16", "given", False), ("f32", "sigmoid", True)])
def test_chains_longer_than_a_tile_looks_back_at_once(apex, dtype, gate, cut):
    """More than 64 stretches of 256 steps in front of the last tile; with factors next to 1 in some channels."""
    c = Scan(2, 20003, 17, dtype, gate, 9, cut, True)
    c.g[:, :, 3] = 9.0 if gate == "sigmoid" else 1.0
    c.g[:, :, 4] = 1.0 if gate == "given" else 7.0
    c.x[:, :, 3:5] *= 0.01
    got = c.run(apex)
    c.check(got, [0, 1], list(range(17)))
