"""The operators around the memory on the GPU, through the binding, against the 64-bit plain forms.  Bounds come from the plain
forms' error recurrences (32-bit arithmetic) and one rounding to the output's type."""
import itertools

import numpy as np
import pytest
import torch

import operators_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NAN = float("nan")


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def to_dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t if dtype is None else t.to(dtype)


def check(got, want, err, dtype, what):
    got = plain.f64(got)
    bound = err + plain.rounding(want, dtype)
    off = np.abs(got - want)
    assert got.shape == want.shape and np.array_equal(np.isnan(got), np.isnan(want)), what
    bad = ~(off <= bound) & ~np.isnan(want) & ~((got == want) & np.isinf(want))
    assert not bad.any(), "%s: %d of %d off, first at %s: %g for %g, bound %g" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], bound[bad][0])


# -------------------------------------------------------------------------------------------------------------- scan

class Scan:
    def __init__(self, S, T, D, dtype, gate, seed=0, cut=False, ragged=False, start=True, last=True, shape=None):
        rng = np.random.default_rng(seed)
        self.S, self.T, self.D, self.dtype, self.gate = S, T, D, DTYPES[dtype], gate
        g = rng.standard_normal((S, T, D)) * 2 + 1 if gate == "sigmoid" else rng.uniform(-0.3, 1.0, (S, T, D))
        self.g, self.x, self.dh = (to_dev(a, self.dtype) for a in (g, rng.standard_normal((S, T, D)), rng.standard_normal((S, T, D))))
        self.h0 = to_dev(rng.standard_normal((S, D)).astype(np.float32)) if start else None
        self.dh_last = to_dev(rng.standard_normal((S, D)).astype(np.float32)) if last else None
        self.discount = to_dev(np.where(rng.random((S, T)) < 0.06, 0.0, 0.99).astype(np.float32)) if cut else None
        length = rng.integers(0, T + 1, S)
        length[0] = T
        if S > 1:
            length[1] = 0
        self.length = to_dev(length.astype(np.int32)) if ragged else None

    def want(self):
        host = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        return plain.scan(plain.f64(self.g), plain.f64(self.x), self.gate, host(self.discount), host(self.length), plain.f64(self.h0),
                          plain.f64(self.dh), plain.f64(self.dh_last))

    def run(self, apex, workspace=None, g=None, x=None, **k):
        g, x = self.g if g is None else g, self.x if x is None else x
        rc, out = apex.gated_scan(g, x, gate=self.gate, discount=self.discount, length=self.length, h0=self.h0, carry=True,
                                  workspace=workspace, **k)
        assert rc == apex.OK
        rc, back = apex.gated_scan_backward(g, x, self.dh, out["carry"], gate=self.gate, discount=self.discount, length=self.length,
                                            dh_last=self.dh_last, workspace=workspace, **k)
        assert rc == apex.OK
        torch.cuda.synchronize()
        return {**out, **back}

    def check(self, got, want=None):
        want = want or self.want()
        for n in ("h", "dg", "dx"):
            check(got[n], want[n], want[n + "_err"], self.dtype, n)
        for n in ("h_last", "dh0"):
            check(got[n], want[n], want[n + "_err"], torch.float32, n)


SHAPES = [(1, 1, 1), (3, 1, 64), (2, 2, 7), (2, 3, 130), (4, 15, 33), (3, 16, 256), (2, 63, 5), (2, 64, 16), (3, 65, 17), (1, 127, 131),
          (2, 128, 128), (2, 129, 100), (3, 200, 72), (1, 257, 1003), (5, 96, 520), (2, 1000, 33), (1, 2049, 40), (1, 5000, 24)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype,gate,cut,ragged", [("f32", "sigmoid", True, True), ("bf16", "sigmoid", False, True),
                                                   ("f16", "given", True, False), ("bf16", "given", True, True),
                                                   ("f32", "given", False, False)])
def test_scan(apex, shape, dtype, gate, cut, ragged):
    c = Scan(*shape, dtype, gate, seed=sum(shape), cut=cut, ragged=ragged, start=shape[0] != 3, last=shape[0] != 4)
    c.check(c.run(apex))


def test_scan_many_sequences(apex):
    for S, T, D in ((300, 5, 3), (700, 70, 9), (65, 130, 64)):
        c = Scan(S, T, D, "bf16", "sigmoid", seed=S, cut=True, ragged=True)
        c.check(c.run(apex))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T", [1, 5, 150])
def test_scan_strides_and_addresses(apex, dtype, T):
    """Halves of one projection, time-major arrays, arrays that begin one element after an aligned address, and an input that is
    broadcast over the sequences; gradients into strided arrays, and in place."""
    S, D = 3, 37
    c = Scan(S, T, D, dtype, "sigmoid", seed=T, cut=True)
    want = c.want()
    both = torch.full((S, T, 2 * D + 1), NAN, dtype=c.dtype, device="cuda:0")
    both[:, :, 1:D + 1], both[:, :, D + 1:] = c.g, c.x
    c.check(c.run(apex, g=both[:, :, 1:D + 1], x=both[:, :, D + 1:]), want)
    turned = torch.empty((T, S, D), dtype=c.dtype, device="cuda:0").copy_(c.g.transpose(0, 1)).transpose(0, 1)
    got = c.run(apex, g=turned)
    c.check(got, want)
    # into the halves of one array, beside which nothing is written, and over the inputs
    grads = torch.full((S, T, 2 * D + 3), 7.0, dtype=c.dtype, device="cuda:0")
    back = dict(dg=grads[:, :, 1:D + 1], dx=grads[:, :, D + 2:2 * D + 2], dh0=torch.empty((S, D), device="cuda:0"))
    k = dict(gate=c.gate, discount=c.discount, dh_last=c.dh_last)
    assert apex.gated_scan_backward(c.g, c.x, c.dh, got["carry"], out=back, **k)[0] == apex.OK
    c.check({**got, **back}, want)
    assert (grads[:, :, [0, D + 1, 2 * D + 2]] == 7.0).all()
    g, x = c.g.clone(), c.x.clone()
    assert apex.gated_scan_backward(g, x, c.dh, got["carry"], out=dict(dg=g, dx=x), **k)[0] == apex.OK
    c.check({**got, "dg": g, "dx": x}, want)
    # one input row set for all sequences
    c.x = c.x[:1].contiguous().expand(S, T, D)
    c.check(c.run(apex))
    if T > 1:
        with pytest.raises(AssertionError):
            apex.gated_scan(c.g.transpose(1, 2), c.x.transpose(1, 2))


def test_scan_state_in_place_and_in_pieces(apex):
    """A sequence in pieces, the state handed on in one buffer, ends where the whole one does; token by token too."""
    c = Scan(4, 150, 40, "f32", "sigmoid", cut=True)
    want = c.want()
    for pieces in ([70, 1, 79], [1] * 150):
        state, h, t = c.h0.clone(), [], 0
        for n in pieces:
            rc, out = apex.gated_scan(c.g[:, t:t + n], c.x[:, t:t + n], discount=c.discount[:, t:t + n].contiguous(), h0=state,
                                      out=dict(h=torch.empty((4, n, 40), device="cuda:0"), h_last=state))
            assert rc == apex.OK
            h.append(out["h"])
            t += n
        torch.cuda.synchronize()
        check(torch.cat(h, 1), want["h"], 2 * want["h_err"], torch.float32, "h in pieces")
        check(state, want["h_last"], 2 * want["h_last_err"], torch.float32, "state in pieces")


@pytest.mark.parametrize("T", [9, 64, 300])
def test_scan_keeps_out_what_is_masked(apex, T):
    """NaN and infinities behind a sequence's length, in a start state that no step takes, and in an episode that has ended."""
    S, D = 4, 24
    c = Scan(S, T, D, "f32", "sigmoid", ragged=True, seed=T)
    cut = T // 2
    discount = np.ones((S, T), np.float32)
    discount[:, cut] = 0.0
    c.length = to_dev(np.array([T, 0, max(1, T // 3), T - 1], np.int32))
    c.discount = to_dev(discount)
    for s, n in enumerate((T, 0, max(1, T // 3), T - 1)):
        for a in (c.g, c.x, c.dh):
            a[s, n:] = NAN if s % 2 else float("inf")
    clean = c.want()
    got = c.run(apex)
    c.check(got, clean)
    for n in ("h", "dg", "dx"):
        assert (got[n][1] == 0).all() and torch.isfinite(got[n]).all(), n
    # an episode full of NaN, then another: only the first one's own steps show it
    c.x[0, :cut + 1] = NAN
    got = c.run(apex)
    assert torch.isnan(got["h"][0, :cut + 1]).all()
    check(got["h"][0, cut + 1:], clean["h"][0, cut + 1:], clean["h_err"][0, cut + 1:], torch.float32, "h behind")
    check(got["dx"][0, cut + 1:], clean["dx"][0, cut + 1:], clean["dx_err"][0, cut + 1:], torch.float32, "dx behind")
    check(got["h_last"], clean["h_last"], clean["h_last_err"], torch.float32, "h_last")
    # and gradients that are NaN behind the episode's end stay there
    c = Scan(S, T, D, "f32", "sigmoid", seed=T)
    c.discount = to_dev(discount)
    clean = c.want()
    c.dh[:, cut + 1:] = NAN
    got = c.run(apex)
    check(got["dx"][:, :cut + 1], clean["dx"][:, :cut + 1], clean["dx_err"][:, :cut + 1], torch.float32, "dx before")
    check(got["dh0"], clean["dh0"], clean["dh0_err"], torch.float32, "dh0")


def test_scan_a_nan_stays_in_its_sequence_and_channel(apex):
    for T in (40, 700):
        c = Scan(3, T, 20, "bf16", "given", seed=1)
        c.g.mul_(0.1)                                     # products over a chunk are below any number: a NaN passes all the same
        c.x[1, 3, 5] = NAN
        got = c.run(apex)
        bad = torch.zeros_like(got["h"], dtype=torch.bool)
        bad[1, 3:, 5] = True
        assert torch.equal(torch.isnan(got["h"]), bad)


def test_scan_same_bits_whatever_else_uses_the_workspace(apex):
    """One workspace for calls of several sizes in turn, with other calls between: every repetition gives the same bits."""
    cases = [Scan(*s, "bf16", "sigmoid", seed=i, cut=True, ragged=True) for i, s in
             enumerate([(3, 1000, 200), (1, 4000, 24), (40, 96, 300), (2, 64, 9), (2, 1, 33)])]
    biggest = [apex.gated_scan_workspace(c.S, c.T, c.D) for c in cases]
    biggest = max((w for w in biggest if w is not None), key=lambda w: w.numel(), default=None)
    first = [c.run(apex, workspace=biggest) for c in cases]
    for _ in range(6):
        for c, f in zip(cases, first):
            got = c.run(apex, workspace=biggest)
            for n in ("h", "h_last", "dg", "dx", "dh0"):
                assert torch.equal(got[n].view(torch.uint8), f[n].view(torch.uint8)), (n, c.S, c.T, c.D)
    for c, f in zip(cases, first):
        c.check(f)


# ----------------------------------------------------------------------------------------------------------- distill

class Distill:
    def __init__(self, N, V, K, dtype, vtype="f32", rest=False, tau=1.0, weighted=True, seed=0, spread=2.0):
        rng = np.random.default_rng(seed)
        self.N, self.V, self.K, self.dtype, self.tau = N, V, K, DTYPES[dtype], tau
        z = rng.standard_normal((N, V)) * spread
        t = z + rng.standard_normal((N, V)) * 0.7
        index = np.argsort(-t, axis=1)[:, :K]
        self.logits = to_dev(z, self.dtype)
        self.index = to_dev(index.astype(np.int32))
        self.value = to_dev(np.take_along_axis(t, index, 1), DTYPES[vtype])
        lse = np.log(np.exp(t / tau).sum(1))
        self.top_lse = to_dev(lse.astype(np.float32)) if rest else None
        self.weight = to_dev(rng.uniform(0.1, 1.0, N).astype(np.float32)) if weighted else None

    def want(self):
        return plain.distill(plain.f64(self.logits), self.index.cpu().numpy(), plain.f64(self.value), float(np.float32(self.tau)),
                             plain.f64(self.top_lse), plain.f64(self.weight))

    def run(self, apex, **k):
        rc, out = apex.distill_topk(self.logits, self.index, self.value, weight=self.weight, top_lse=self.top_lse, temperature=self.tau, **k)
        assert rc == apex.OK
        torch.cuda.synchronize()
        return out

    def check(self, got, want=None):
        want = want or self.want()
        check(got["loss"], want["loss"], want["loss_err"], torch.float32, "loss")
        if got.get("lse") is not None:
            check(got["lse"], want["lse"], want["lse_err"], torch.float32, "lse")
        if got.get("grad") is not None:
            check(got["grad"], want["grad"], want["grad_err"], self.dtype, "grad")


@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (2, 2, 2), (3, 7, 3), (5, 8, 8), (4, 65, 17), (2, 513, 64), (3, 1000, 1000), (7, 4096, 33),
                                   (2, 5003, 129), (1, 20011, 1024), (3, 32768, 64), (2, 49999, 17), (1, 131072, 128), (1, 262147, 5)])
@pytest.mark.parametrize("dtype,rest,tau", [("f32", False, 1.0), ("f32", True, 2.5), ("bf16", True, 1.0), ("bf16", False, 1.5),
                                            ("f16", False, 1.0), ("f16", True, 1.0)])
def test_distill(apex, N, V, K, dtype, rest, tau):
    c = Distill(N, V, K, dtype, vtype=("f32", "bf16", "f16")[(N + K) % 3], rest=rest, tau=tau, weighted=N != 3, seed=V)
    got = c.run(apex)
    want = c.want()
    c.check(got, want)
    c.check(c.run(apex, grad=False), want)


@pytest.mark.parametrize("N,V", [(300, 1003), (700, 300), (1500, 130), (260, 9001)])
def test_distill_many_rows(apex, N, V):
    c = Distill(N, V, 9, "bf16", rest=N % 2 == 0, seed=N)
    c.check(c.run(apex))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,V", [(2, 33), (3, 4099), (2, 70001), (600, 77)])
def test_distill_strides_and_in_place(apex, dtype, N, V):
    """A padded vocabulary from an odd address, whose padding holds NaN and stays as it is; the gradient in place."""
    c = Distill(N, V, 11, dtype, rest=True, seed=N)
    want = c.want()
    held = torch.full((N, V + 9), NAN, dtype=c.dtype, device="cuda:0")
    held[:, 3:V + 3] = c.logits
    c.logits = held[:, 3:V + 3]
    c.check(c.run(apex), want)
    out = dict(loss=torch.empty(N, device="cuda:0"), grad=c.logits)
    c.check(c.run(apex, out=out), want)
    assert torch.isnan(held[:, :3]).all() and torch.isnan(held[:, V + 3:]).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V", [50, 3001, 40000])
def test_distill_places_that_do_not_count(apex, rest, V):
    """Empty places (whatever their value), indices out of range, tokens named twice, rows that name nothing, values of -inf,
    logits of -inf among the named and the others, rows of weight 0."""
    c = Distill(9, V, 6, "f32", rest=rest, seed=V)
    c.index[0, 2], c.value[0, 2] = -1, NAN
    c.index[1, 0], c.value[1, 0], c.index[1, 5], c.value[1, 5] = V, float("inf"), -2147483648, NAN
    c.index[2, 3], c.value[2, 3] = c.index[2, 1], 50.0          # named twice: the first place counts
    c.index[3], c.value[3] = -1, NAN                             # names nothing
    c.value[4, 1] = -float("inf")
    c.logits[5, c.index[5, 0].item()] = -float("inf")            # the teacher's first token is impossible: the loss is infinite
    c.logits[6][c.logits[6] < 0] = -float("inf")                 # a mask over the vocabulary
    c.logits[6, c.index[6].long()] = 1.0
    c.weight[7] = 0.0
    c.logits[8] = -float("inf")
    c.logits[8, c.index[8].long()] = 0.5                         # all others impossible
    if rest:
        c.top_lse[8] = float(torch.logsumexp(c.value[8].double(), 0)) + 1e-3
    got, want = c.run(apex), c.want()
    assert float(want["loss"][5]) == np.inf and float(want["loss"][3]) == 0
    assert not rest or float(want["loss"][8]) == np.inf
    c.check(got, want)
    assert (got["grad"][3].abs() <= 1e-7).all() and (got["grad"][7] == 0).all()
    # rows that have no answer say so, and leave the others alone
    c.logits[0, V // 2] = NAN
    c.logits[1, 0] = float("inf")
    c.logits[2] = -float("inf")
    c.value[4, 1] = NAN
    c.logits[7, 1] = NAN                                         # of weight 0: no gradient all the same
    bad = c.run(apex)
    for i in (0, 1, 2, 4):
        assert torch.isnan(bad["loss"][i]) and torch.isnan(bad["grad"][i]).any(), i
    assert torch.isnan(bad["loss"][7]) and (bad["grad"][7] == 0).all()
    for i in (3, 5, 6, 8):
        assert torch.equal(bad["loss"][i], got["loss"][i]) and torch.equal(bad["grad"][i], got["grad"][i]), i


def test_distill_far_apart(apex):
    """Logits of the size of hundreds, and a student that gives the rest next to nothing: no overflow, and the rest's share
    keeps its precision."""
    for spread in (30.0, 300.0):
        for rest in (False, True):
            c = Distill(4, 5000, 8, "f32", rest=rest, seed=1, spread=spread)
            c.check(c.run(apex))
    c = Distill(3, 4000, 4, "f32", rest=True, seed=2, spread=1.0)
    c.logits.scatter_add_(1, c.index.long(), torch.full((3, 4), 60.0, device="cuda:0"))
    got, want = c.run(apex), c.want()
    assert (want["loss"] > 10).all()
    c.check(got, want)


def test_distill_same_bits(apex):
    for N, V, K in ((3, 60001, 100), (600, 2000, 1000)):
        c = Distill(N, V, K, "bf16", rest=True, seed=N)
        first = c.run(apex)
        for _ in range(5):
            got = c.run(apex)
            for n in ("loss", "lse", "grad"):
                assert torch.equal(got[n], first[n]), n


# ------------------------------------------------------------------------------------------------------------ verify

class Verify:
    def __init__(self, B, G, V, dtype, ragged=False, seed=0, noise=0.5):
        rng = np.random.default_rng(seed)
        z = rng.standard_normal((B, G + 1, V)) * 2

        def soft(a):
            a = np.exp(a - a.max(2, keepdims=True))
            return a / a.sum(2, keepdims=True)
        self.target = to_dev(soft(z + rng.standard_normal(z.shape) * noise), DTYPES[dtype])
        self.draft = to_dev(soft(z[:, :G]), DTYPES[dtype]) if G else None
        self.token = None
        if G:
            up_to = soft(z[:, :G]).cumsum(2)
            self.token = to_dev((up_to < rng.random((B, G, 1)) * up_to[:, :, -1:]).sum(2).clip(max=V - 1).astype(np.int32))
        self.rnd = to_dev(rng.integers(0, 1 << 64, (B, G + 1), dtype=np.uint64).view(np.int64))
        self.length = to_dev(rng.integers(-1, G + 2, B).astype(np.int32)) if ragged else None

    def check(self, apex, workspace=None, **k):
        host = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        d = self.draft if self.draft is not None else torch.zeros((self.target.shape[0], 0, self.target.shape[2]))
        want = plain.verify(plain.f64(self.target), plain.f64(d), host(self.token), host(self.rnd).view(np.uint64), host(self.length))
        rc, out = apex.verify_draft(self.target, self.draft, self.token, self.rnd, length=self.length, workspace=workspace, **k)
        assert rc == apex.OK
        torch.cuda.synchronize()
        assert np.array_equal(host(out["accepted"]), want[0])
        assert np.array_equal(host(out["token"]), want[1])
        return want


@pytest.mark.parametrize("B,G,V", [(1, 1, 1), (3, 2, 2), (5, 4, 9), (300, 3, 64), (2, 64, 100), (1, 5, 4095), (4, 3, 4097), (70, 8, 1000),
                                   (1, 4, 50021), (3, 2, 131072), (1, 1, 300007), (4, 0, 777), (1300, 1, 33)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_verify(apex, B, G, V, dtype):
    for ragged in (False, True) if G else (False,):
        for noise in (0.0, 0.5, 3.0):
            Verify(B, G, V, dtype, ragged, seed=B + V, noise=noise).check(apex)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_verify_edges(apex, dtype):
    """Uniforms at both ends, equal distributions (nothing is left: the target's own row is drawn from), certain tokens, rows without
    mass, NaN, negative and infinite probabilities, tokens out of range, masses that no 2^-40 reaches."""
    B, G, V = 12, 3, 5000
    c = Verify(B, G, V, dtype, seed=7)
    c.rnd[0], c.rnd[1] = 0, -1
    c.draft[2] = c.target[2, :G]
    c.rnd[2] = -1                                    # equal: all stand, even so
    c.draft[3, 1] = c.target[3, 1]
    c.token[3, 1] = V                                # out of range: turned down, nothing is left
    c.target[4, 0] = 0
    c.target[4, 0, V - 1] = 1                        # the last token, for certain
    c.target[5, 0] = 0                               # no mass
    c.target[6, 0] = NAN
    c.target[6, 0, 17] = float("inf")
    c.target[7, 0] = -1.0
    c.target[7, 0, 4321] = 2.0
    c.draft[8, 0] = NAN                              # a draft without mass
    c.token[9, 0] = -5
    c.target[10, 0] = 1e-13 if dtype != "f16" else 0.0
    c.target[10, 0, 99] = 1e-11 if dtype != "f16" else 6e-8
    c.draft[11] = 0
    c.draft[11, :, 3] = 1
    c.token[11] = 3
    c.target[11] = 0
    c.target[11, :, 3] = 1                           # both certain: everything stands, and the bonus is the same
    accepted, token = c.check(apex)
    assert accepted[2] == 3 and accepted[3] <= 1 and token[5, 0] == -1 and token[11].tolist() == [3] * 4


def test_verify_sums_that_no_normalised_row_reaches(apex):
    """Every probability 1 (weights that nobody normalised), in so many sequences that a row has one or two workgroups: sums of
    2^60, and what is drawn is uniform in the uniforms."""
    rng = np.random.default_rng(8)
    for B, V in ((5000, 1 << 20), (4100, (1 << 19) + 5)):
        row = torch.ones((1, 2, V), dtype=torch.bfloat16, device="cuda:0")
        row[:, :, 0] = 7.0
        rnd = rng.integers(0, 1 << 64, (B, 2), dtype=np.uint64)
        token = to_dev(np.full((B, 1), -1, np.int32))
        rc, out = apex.verify_draft(row.expand(B, 2, V), torch.zeros((1, 1, V), dtype=torch.bfloat16, device="cuda:0").expand(B, 1, V),
                                    token, to_dev(rnd.view(np.int64)))
        assert rc == apex.OK
        torch.cuda.synchronize()
        want = np.array([(int(u) * (V << 40)) >> 104 for u in rnd[:, 1]])
        assert (out["accepted"] == 0).all() and np.array_equal(out["token"][:, 0].cpu().numpy(), want)


def test_verify_strides_addresses_and_workspace(apex):
    """Padded rows from odd addresses, one target row for all places, a workspace that calls of several sizes share."""
    space = apex.verify_draft_workspace(80, 20000)
    for dtype, (B, G, V) in itertools.product(DTYPES, ((2, 3, 9001), (80, 1, 333), (1, 2, 20000), (7, 5, 4096))):
        c = Verify(B, G, V, dtype, ragged=True, seed=V)
        t = torch.full((B, G + 1, V + 5), NAN, dtype=c.target.dtype, device="cuda:0")
        d = torch.full((G, B, V + 2), NAN, dtype=c.target.dtype, device="cuda:0")
        t[:, :, 1:V + 1], d[:, :, 1:V + 1] = c.target, c.draft.transpose(0, 1)
        c.target, c.draft = t[:, :, 1:V + 1], d.transpose(0, 1)[:, :, 1:V + 1]
        for _ in range(3):
            c.check(apex, workspace=space)
        c.target = c.target[:, :1].expand(B, G + 1, V)
        c.check(apex, workspace=space)


# ---------------------------------------------------------------------------------------------- far apart, and the largest

def test_rows_whose_offsets_pass_32_bits(apex):
    """Rows 2^31 and more elements apart (13 GB of bf16, of which only the rows are filled)."""
    far = (1 << 31) + 24
    held = torch.empty((3, far), dtype=torch.bfloat16, device="cuda:0")
    c = Distill(3, 2003, 7, "bf16", rest=True, seed=3)
    want = c.want()
    held[:, 8:2011] = c.logits
    c.logits = held[:, 8:2011]
    c.check(c.run(apex, out=dict(loss=torch.empty(3, device="cuda:0"), grad=c.logits)), want)
    s = Scan(3, 150, 40, "bf16", "sigmoid", seed=4, cut=True)
    want = s.want()
    rows = torch.as_strided(held, (3, 150, 40), (far, 64, 1))
    rows.copy_(s.g)
    s.check(s.run(apex, g=rows), want)
    v = Verify(3, 1, 4000, "bf16", seed=5)
    t = torch.as_strided(held, (3, 2, 4000), (far, 4096, 1))
    t.copy_(v.target)
    v.target = t
    v.check(apex)
    v.target = t.contiguous()
    d = torch.as_strided(held, (3, 1, 4000), (far, 1, 1), storage_offset=16)
    d.copy_(v.draft)
    v.draft = d
    v.check(apex)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_largest_vocabulary(apex, dtype):
    c = Distill(2, apex.MAX_VOCABULARY, apex.MAX_TOP, dtype, rest=True, seed=6)
    c.check(c.run(apex))
    Verify(2, 2, apex.MAX_VOCABULARY, dtype, seed=7).check(apex)


# -------------------------------------------------------------------------------------------------- streams and graphs

def test_operators_on_a_stream_of_their_own_and_in_a_graph(apex):
    """Every operator on a side stream behind work that makes its inputs there, then recorded once and replayed over new inputs,
    with other work in between: each replay equals the plain call on the same inputs."""
    s, d, v = (Scan(3, 700, 50, "bf16", "sigmoid", cut=True, ragged=True), Distill(40, 9001, 12, "bf16", rest=True),
               Verify(6, 3, 9001, "f32", ragged=True))
    spaces = apex.gated_scan_workspace(3, 700, 50), apex.distill_topk_workspace(40, 9001), apex.verify_draft_workspace(6, 9001)

    def outputs():
        return (dict(h=torch.empty_like(s.x), h_last=torch.empty((3, 50), device="cuda:0"),
                     carry=torch.empty(apex.gated_scan_carry_shape(3, 700, 50), device="cuda:0")),
                dict(dg=torch.empty_like(s.g), dx=torch.empty_like(s.x), dh0=torch.empty((3, 50), device="cuda:0")),
                dict(loss=torch.empty(40, device="cuda:0"), lse=torch.empty(40, device="cuda:0"), grad=torch.empty_like(d.logits)),
                dict(accepted=torch.empty(6, dtype=torch.int32, device="cuda:0"), token=torch.empty((6, 4), dtype=torch.int32, device="cuda:0")))

    def calls(out):
        assert apex.gated_scan(s.g, s.x, discount=s.discount, length=s.length, h0=s.h0, out=out[0], workspace=spaces[0])[0] == 0
        assert apex.gated_scan_backward(s.g, s.x, s.dh, out[0]["carry"], discount=s.discount, length=s.length, dh_last=s.dh_last,
                                        out=out[1], workspace=spaces[0])[0] == 0
        assert apex.distill_topk(d.logits, d.index, d.value, weight=d.weight, top_lse=d.top_lse, out=out[2], workspace=spaces[1])[0] == 0
        assert apex.verify_draft(v.target, v.draft, v.token, v.rnd, length=v.length, out=out[3], workspace=spaces[2])[0] == 0

    def equal(a, b):
        for x, y in zip(a, b):
            for n in x:
                if n != "carry":
                    assert torch.equal(x[n], y[n]), n

    plainly, recorded = outputs(), outputs()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.x.mul_(0.5)
        d.logits.mul_(0.5)
        calls(plainly)
    side.synchronize()
    s.check({**plainly[0], **plainly[1]})
    d.check(plainly[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(recorded)
    for i in range(5):
        s.x.add_(0.1)
        d.logits.add_(torch.randn_like(d.logits))
        v.rnd.add_(1 << 60)
        graph.replay()
        torch.randn(1000, 1000, device="cuda:0").sum().item()
        calls(plainly)
        torch.cuda.synchronize()
        equal(recorded, plainly)


def test_operators_on_a_stream_that_is_not_the_current_one(apex):
    """stream= without outputs and workspace, while the current stream uses and gives back memory of the same sizes: what the
    calls make for themselves belongs to their stream."""
    s, d, v = Scan(2, 900, 60, "f32", "sigmoid", cut=True), Distill(30, 5001, 9, "f32", rest=True), Verify(5, 3, 70001, "f32")
    host = lambda t: t.cpu().numpy()  # noqa: E731
    wants = s.want(), d.want(), plain.verify(plain.f64(v.target), plain.f64(v.draft), host(v.token), host(v.rnd).view(np.uint64))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        for n in (5 * 1152, 30 * 4, 30 * 5001 * 4, 2 * 900 * 60 * 4):
            used = torch.full((n,), 255, dtype=torch.uint8, device="cuda:0")
            used.fill_(255)
            del used
        rc, out = apex.gated_scan(s.g, s.x, discount=s.discount, h0=s.h0, carry=True, stream=side)
        assert rc == apex.OK
        rc, back = apex.gated_scan_backward(s.g, s.x, s.dh, out["carry"], discount=s.discount, dh_last=s.dh_last, stream=side)
        assert rc == apex.OK
        rc, loss = apex.distill_topk(d.logits, d.index, d.value, weight=d.weight, top_lse=d.top_lse, stream=side)
        assert rc == apex.OK
        rc, verdict = apex.verify_draft(v.target, v.draft, v.token, v.rnd, stream=side)
        assert rc == apex.OK
        side.synchronize()
        s.check({**out, **back}, wants[0])
        d.check(loss, wants[1])
        assert np.array_equal(host(verdict["accepted"]), wants[2][0]) and np.array_equal(host(verdict["token"]), wants[2][1])
