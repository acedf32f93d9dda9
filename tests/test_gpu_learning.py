"""Gated delta rule, embedding and clipped gradients on the GPU, through the binding, against the 64-bit plain forms.  Bounds come
from the plain forms' magnitudes (32-bit sums of products) and one rounding to the output's type."""
import numpy as np
import pytest
import torch

import learning_plain as plain
from operators_plain import rounding

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NAN = float("nan")
BACK = ("dq", "dk", "dv", "dg", "dbeta", "dh0")


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def to_dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t if dtype is None else t.to(dtype)


def check(got, want, err, dtype, what):
    got = plain.f64(got)
    assert got.shape == want.shape, what
    off = np.abs(got - want)
    bad = ~(off <= np.broadcast_to(err, want.shape) + rounding(want, dtype))
    assert not bad.any(), "%s: %d of %d off, first at %s: %g for %g, bound %g" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], (np.broadcast_to(err, want.shape) + rounding(want, dtype))[bad][0])


# ------------------------------------------------------------------------------------------------------- delta rule

class Delta:
    def __init__(self, S, T, Hk, H, Dk, Dv, dtype, seed=0, cut=False, ragged=False, start=True, last=True, alike=0.0, strength=None):
        rng = np.random.default_rng(seed)
        self.sizes, self.dtype, self.scale = (S, T, Hk, H, Dk, Dv), DTYPES[dtype], Dk ** -0.5
        same = rng.standard_normal((1, 1, Hk, Dk)) * alike
        q, k = (rng.standard_normal((S, T, Hk, Dk)) + same for _ in range(2))
        q, k = (x / np.maximum(np.sqrt((x ** 2).sum(3, keepdims=True)), 1e-6) * (1 - 2.0 ** -7) for x in (q, k))
        self.q, self.k, self.v, self.do = (to_dev(x, self.dtype) for x in (q, k, rng.standard_normal((S, T, H, Dv)), rng.standard_normal((S, T, H, Dv))))
        g = -np.exp(rng.standard_normal((S, T, H)) * 1.5 - 3.0)
        beta = 1 / (1 + np.exp(-2 * rng.standard_normal((S, T, H)))) if strength is None else np.full((S, T, H), strength)
        self.g, self.beta = to_dev(g.astype(np.float32)), to_dev(beta.astype(np.float32))
        self.h0 = to_dev(rng.standard_normal((S, H, Dk, Dv)).astype(np.float32)) if start else None
        self.dh_last = to_dev(rng.standard_normal((S, H, Dk, Dv)).astype(np.float32)) if last else None
        self.discount = to_dev(np.where(rng.random((S, T)) < 0.06, 0.0, 0.99).astype(np.float32)) if cut else None
        length = rng.integers(0, T + 1, S)
        length[0] = T
        if S > 1:
            length[1] = 0
        self.length = to_dev(length.astype(np.int32)) if ragged else None

    def want(self):
        host = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        opt = lambda t: None if t is None else plain.f64(t)  # noqa: E731
        return plain.delta(plain.f64(self.q), plain.f64(self.k), plain.f64(self.v), plain.f64(self.g), plain.f64(self.beta), self.scale,
                           host(self.discount), host(self.length), opt(self.h0), plain.f64(self.do), opt(self.dh_last))

    def run(self, apex, workspace=None, **k):
        given = {n: k.pop(n, getattr(self, n)) for n in ("q", "k", "v", "do")}
        back = k.pop("back", None)
        more = dict(discount=self.discount, length=self.length, scale=self.scale, workspace=workspace, **k)
        rc, out = apex.delta_rule(given["q"], given["k"], given["v"], self.g, self.beta, h0=self.h0, carry=True, **more)
        assert rc == apex.OK
        rc, back = apex.delta_rule_backward(given["q"], given["k"], given["v"], self.g, self.beta, given["do"], out["carry"], dh_last=self.dh_last,
                                            out=back, **more)
        assert rc == apex.OK
        torch.cuda.synchronize()
        return {**out, **back}

    def check(self, got, want=None, names=("o", "h_last") + BACK):
        want = want or self.want()
        _, _, _, _, Dk, Dv = self.sizes
        for n in names:
            bound = plain.delta_bound(n, want, Dk, Dv)
            if n in ("dg", "dbeta"):
                bound = bound[..., 0]
            check(got[n], want[n], bound, torch.float32 if n in ("h_last", "dg", "dbeta", "dh0") else self.dtype, n)


SHAPES = [(1, 1, 1, 1, 1, 1), (3, 1, 2, 4, 128, 128), (2, 5, 1, 3, 12, 70), (2, 8, 1, 2, 30, 64), (2, 9, 1, 2, 70, 64), (2, 16, 2, 2, 65, 3), (2, 17, 1, 2, 16, 16), (3, 63, 1, 1, 33, 47),
          (2, 64, 2, 2, 64, 64), (2, 65, 1, 2, 100, 128), (1, 129, 2, 6, 128, 20), (3, 200, 1, 1, 17, 33), (1, 513, 1, 2, 128, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype,cut,ragged", [("f32", True, True), ("bf16", False, True), ("f16", True, False), ("bf16", True, True), ("f32", False, False)])
def test_delta(apex, shape, dtype, cut, ragged):
    c = Delta(*shape, dtype, seed=sum(shape), cut=cut, ragged=ragged, start=shape[0] != 3, last=shape[4] != 100)
    c.check(c.run(apex))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_delta_many_sequences(apex, dtype):
    # (the last one: more slices of 16 columns than compute units, an odd number a head)
    for shape in ((70, 3, 2, 2, 16, 40), (130, 16, 2, 2, 20, 70), (90, 70, 1, 4, 32, 96), (300, 20, 1, 1, 8, 8), (20, 70, 1, 2, 72, 100), (9, 130, 4, 4, 128, 128)):
        c = Delta(*shape, dtype, seed=shape[0], cut=True, ragged=True)
        c.check(c.run(apex))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_delta_of_a_sequence_does_not_depend_on_how_many_there_are(apex, dtype):
    """Many sequences share a workgroup's columns, and f16 keys are held otherwise than for few; every product is the same."""
    S, T, Hk, H, Dk, Dv = 9, 150, 2, 4, 104, 120  # 9 * 4 * 8 slices of 16 columns: more than compute units
    d = Delta(S, T, Hk, H, Dk, Dv, dtype, cut=True, ragged=True)
    every = d.run(apex)
    for s in (0, 4):
        part = slice(s, s + 1)
        one = Delta(1, T, Hk, H, Dk, Dv, dtype)
        for n in ("q", "k", "v", "do", "g", "beta", "h0", "dh_last", "discount", "length"):
            setattr(one, n, getattr(d, n)[part])
        alone = one.run(apex)
        for n in ("o", "h_last") + BACK:
            assert torch.equal(alone[n], every[n][part]), (n, s)
    d.check(every)


@pytest.mark.parametrize("strength", [0.0, 1.0, 2.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_delta_keys_that_are_nearly_alike(apex, dtype, strength):
    """Where the system that a piece solves is as far from diagonal as it gets; and strengths of 0, for which it has no inverse scale."""
    c = Delta(2, 150, 1, 2, 32, 24, dtype, seed=7, alike=8.0, strength=strength)
    c.check(c.run(apex))


@pytest.mark.parametrize("T", [7, 150])
def test_delta_decays(apex, T):
    """Decays that cut (-inf, and those whose exponential is 0), that nearly do, none at all, and a fast one beside slow ones."""
    c = Delta(2, T, 1, 2, 20, 30, "f32", seed=T)
    g = c.g.clone()
    g[0, 1, 0], g[0, T - 2, 1], g[1, 3, 0], g[1, 4, 1], g[1, 5, 0] = -float("inf"), -1000.0, -80.0, -60.0, -30.0
    g[:, T // 2:, 1] = 0.0
    g[1, 0, 1] = -float("inf")
    c.g = g
    got = c.run(apex)
    c.check(got)
    assert got["dg"][0, 1, 0] == 0.0 and got["dg"][1, 0, 1] == 0.0


@pytest.mark.parametrize("T", [7, 150])
def test_delta_decays_whose_exponential_is_zero(apex, T):
    c = Delta(2, T, 1, 2, 20, 30, "bf16", seed=T)
    c.g = c.g.clone()
    for t in (2, T - 2):
        c.g[0, t, 1] = -1000.0
    got = c.run(apex)
    c.check(got)
    assert got["dg"][0, 2, 1] == 0.0 and got["dg"][0, T - 2, 1] == 0.0 and got["dg"][0, 3, 1] != 0.0


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T", [1, 5, 100])
def test_delta_strides_and_addresses(apex, dtype, T):
    """Parts of one projection that begin an element behind an aligned address, time-major arrays, an input that all sequences share;
    gradients into strided arrays, beside which nothing is written."""
    S, Hk, H, Dk, Dv = 3, 2, 4, 21, 13
    c = Delta(S, T, Hk, H, Dk, Dv, dtype, seed=T, cut=True)
    want = c.want()
    widths = (Hk * Dk, Hk * Dk, H * Dv)
    both = torch.full((S, T, sum(widths) + 1), NAN, dtype=c.dtype, device="cuda:0")
    parts = both[:, :, 1:].split(widths, 2)
    q, k, v = (p.unflatten(2, x.shape[2:]) for p, x in zip(parts, (c.q, c.k, c.v)))
    for p, x in zip((q, k, v), (c.q, c.k, c.v)):
        p.copy_(x)
    grads = torch.full((S, T, sum(widths) + 3), 7.0, dtype=c.dtype, device="cuda:0")
    at = (1, 2 + widths[0], 2 + 2 * widths[0])
    dq, dk, dv = (grads[:, :, a:a + w].unflatten(2, x.shape[2:]) for a, w, x in zip(at, widths, (c.q, c.k, c.v)))
    back = dict(dq=dq, dk=dk, dv=dv, dg=torch.empty_like(c.g), dbeta=torch.empty_like(c.g), dh0=torch.empty_like(c.h0))
    c.check(c.run(apex, q=q, k=k, v=v, back=back), want)
    assert (grads[:, :, [0, 1 + widths[0], grads.shape[2] - 1]] == 7.0).all()
    turned = torch.empty((T, S, Hk, Dk), dtype=c.dtype, device="cuda:0").copy_(c.k.transpose(0, 1)).transpose(0, 1)
    c.check(c.run(apex, k=turned), want)
    c.q = c.q[:1].expand(S, T, Hk, Dk)
    c.check(c.run(apex))


@pytest.mark.parametrize("T", [9, 150])
def test_delta_keeps_out_what_is_masked(apex, T):
    """Steps behind a sequence's length hold NaN and are neither read nor do their gradients hold anything but 0; an ended episode's
    state does not pass, whatever it holds, from one call or piece to the next."""
    c = Delta(3, T, 1, 2, 24, 40, "bf16", seed=T, ragged=True)
    want, clean = c.want(), c.run(apex)
    behind = torch.arange(T, device="cuda:0")[None, :] >= c.length[:, None]
    for x in (c.q, c.k, c.v, c.g, c.beta, c.do):
        x[behind] = NAN
    got = c.run(apex)
    c.check(got, want)
    for n in ("o", "h_last") + BACK:
        assert torch.equal(got[n], clean[n]), n
    for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
        assert (got[n][behind] == 0).all(), n
    assert torch.equal(got["h_last"][1], c.h0[1]) and torch.equal(got["dh0"][1], c.dh_last[1])
    # the first step's decay cuts: h0 may hold anything
    c = Delta(2, T, 1, 1, 8, 8, "f32", seed=T, start=True)
    c.g[:, 0] = -float("inf")
    clean = c.run(apex)
    c.h0 = torch.full_like(c.h0, NAN)
    got = c.run(apex)
    assert torch.equal(got["o"], clean["o"]) and torch.equal(got["h_last"], clean["h_last"])
    # and the last step's end: nothing passes on
    c = Delta(2, T, 1, 1, 8, 8, "f32", seed=T)
    c.discount = torch.ones((2, T), device="cuda:0")
    c.discount[:, -1] = 0.0
    got = c.run(apex)
    assert (got["h_last"] == 0).all()
    c.check(got)
    c.dh_last = torch.full_like(c.dh_last, NAN)
    again = c.run(apex)
    for n in BACK:
        assert torch.equal(got[n], again[n]), n


def test_delta_a_nan_stays_in_its_sequence_and_head(apex):
    for T in (5, 100):
        c = Delta(3, T, 2, 4, 20, 20, "bf16", seed=T)
        clean = c.run(apex)
        c.v[1, 2, 2, 3] = NAN
        got = c.run(apex)
        for n in ("o", "h_last", "dv", "dg", "dbeta", "dh0"):
            heads = 1 if n in ("h_last", "dh0") else 2
            a, b = got[n], clean[n]
            keep = [i for i in range(4) if i != 2]
            assert torch.equal(a[[0, 2]], b[[0, 2]]), n
            assert torch.equal(a.movedim(heads, 0)[keep], b.movedim(heads, 0)[keep]), n
        assert got["o"][1, 2, 2, 3].isnan() and got["h_last"][1, 2, :, 3].isnan().all()
        for n in ("dq", "dk"):
            assert torch.equal(got[n][[0, 2]], clean[n][[0, 2]]) and torch.equal(got[n][1, :, 0], clean[n][1, :, 0]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_delta_state_in_place_and_in_pieces(apex, dtype):
    """A sequence in pieces of any length, the state kept in one buffer, is the sequence at once."""
    c = Delta(2, 300, 1, 2, 40, 50, dtype, seed=4, cut=True)
    want = c.want()
    state, o, at = c.h0.clone(), [], 0
    for n in (1, 64, 3, 100, 16, 1, 17, 98):
        part = slice(at, at + n)
        # (what passed out of the piece before is in the state: a step's own end belongs to its piece)
        rc, out = apex.delta_rule(c.q[:, part], c.k[:, part], c.v[:, part], c.g[:, part].contiguous(), c.beta[:, part].contiguous(), h0=state,
                                  discount=c.discount[:, part].contiguous(), scale=c.scale,
                                  out=dict(o=torch.empty((2, n, 2, 50), dtype=c.dtype, device="cuda:0"), h_last=state))
        assert rc == apex.OK
        o.append(out["o"])
        at += n
    assert at == 300
    c.check(dict(o=torch.cat(o, 1), h_last=state), want, names=("o", "h_last"))
    carry = c.run(apex)["carry"]                                        # [S,chunks,H,4,2,8,4,16]: column / 16, row / 32, row % 8, row / 8 % 4, column % 16
    states = carry.permute(0, 1, 2, 4, 6, 5, 3, 7).reshape(2, 5, 2, 64, 64)
    check(states[..., :40, :50], want["carry"], plain.delta_bound("h_last", want, 40, 50)[:, None], torch.float32, "carry")
    assert (states[..., 40:, :] == 0).all() and (states[..., 50:] == 0).all()


def test_delta_same_bits(apex):
    """Whatever the workspace held, whether a carry is asked for, and again and again."""
    for shape in ((2, 10, 1, 2, 16, 32), (2, 200, 1, 2, 64, 100)):
        c = Delta(*shape, "bf16", seed=1, cut=True, ragged=True)
        S, T, _, H, Dk, Dv = shape
        first = c.run(apex)
        space = apex.delta_rule_workspace(S, T, H, Dk, Dv, backward=True)
        for fill in (0, 255, 77):
            space.fill_(fill)
            got = c.run(apex, workspace=space)
            for n in ("o", "h_last") + BACK:
                assert torch.equal(first[n], got[n]), (n, fill)
        rc, out = apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, h0=c.h0, discount=c.discount, length=c.length, scale=c.scale)
        assert rc == apex.OK and torch.equal(out["o"], first["o"]) and torch.equal(out["h_last"], first["h_last"])


# -------------------------------------------------------------------------------------------------------- embedding

def embed(apex, N, V, D, dtype, seed=0, scale=1.5, tokens=None, pad=0, **k):
    rng = np.random.default_rng(seed)
    dt = DTYPES[dtype]
    table, dout = (to_dev(rng.standard_normal((n, D + pad)), dt)[:, pad:] for n in (V, N))
    token = to_dev((rng.integers(-1, V + 1, N) if tokens is None else tokens).astype(np.int32))
    rc, out = apex.embedding(table, token, scale=scale)
    assert rc == apex.OK
    rc, back = apex.embedding_backward(dout, token, V, scale=scale, **k)
    assert rc == apex.OK
    torch.cuda.synchronize()
    t = token.cpu().numpy()
    check(out["out"], plain.embedding(plain.f64(table), t, scale), abs(plain.embedding(plain.f64(table), t, scale)) * 2.0 ** -24, dt, "out")
    want, err = plain.embedding_backward(plain.f64(dout), t, V, scale)
    check(back["dtable"], want, err, dt, "dtable")
    return table, dout, token, out["out"], back["dtable"]


@pytest.mark.parametrize("N,V,D", [(1, 1, 1), (2, 3, 5), (64, 1, 8), (65, 2, 33), (63, 40, 130), (128, 2047, 16), (1000, 2048, 7), (1025, 3000, 64),
                                   (5000, 70, 257), (4097, 5000, 520), (8192, 9000, 3), (8193, 9, 5), (16384, 9, 24), (16385, 100, 9), (20000, 30000, 12), (70000, 3, 5)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_embedding(apex, N, V, D, dtype):
    embed(apex, N, V, D, dtype, seed=N)


def test_embedding_tokens_that_fill_slices(apex):
    """Runs of a token that end and begin at, before and behind the slices' borders, of 64 and of 4096."""
    for runs in ((64, 64, 128), (63, 65, 1, 63, 64), (1, 127, 64, 4096), (4096, 4096), (4095, 4097, 3), (4100, 8192, 50), (20, 12288, 4096 * 3)):
        tokens = np.repeat(np.arange(len(runs)), runs)
        for order in (tokens, tokens[::-1], np.random.default_rng(0).permutation(tokens)):
            embed(apex, len(order), len(runs) + 2, 19, "f32", tokens=order)


def test_embedding_strides_and_tokens_outside(apex):
    for N, V, D in ((50, 20, 31), (300, 500, 1027)):
        for dtype in DTYPES:
            embed(apex, N, V, D, dtype, pad=3)
    tokens = np.array([-1, 5, 2 ** 31 - 1, -2 ** 31, 4, 0])
    _, _, _, out, grad = embed(apex, 6, 5, 8, "f32", tokens=tokens)
    assert (out[[0, 1, 2, 3]] == 0).all() and (grad[1:4] == 0).all()
    _, _, _, out, grad = embed(apex, 40, 5, 8, "bf16", tokens=np.full(40, -1))
    assert (out == 0).all() and (grad == 0).all()
    _, _, _, out, _ = embed(apex, 40, 5, 8, "f32", tokens=np.full(40, -1), scale=-1.0)
    assert not out.signbit().any()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_embedding_gradient_that_is_added(apex, dtype):
    """To what is there already, where a token is named; into rows of a wider array, beside which nothing is written."""
    N, V, D = 700, 90, 45
    rng = np.random.default_rng(2)
    dout = to_dev(rng.standard_normal((N, D)), DTYPES[dtype])
    token = to_dev(rng.integers(-1, 60, N).astype(np.int32))
    held = to_dev(rng.standard_normal((V, D + 4)), DTYPES[dtype])
    had = held.clone()
    rc, out = apex.embedding_backward(dout, token, V, scale=0.5, add=True, out=dict(dtable=held[:, 2:2 + D]))
    assert rc == apex.OK
    want, err = plain.embedding_backward(plain.f64(dout), token.cpu().numpy(), V, 0.5)
    want += plain.f64(had[:, 2:2 + D])
    check(out["dtable"], want, err + abs(want) * 2.0 ** -24, DTYPES[dtype], "dtable")
    assert torch.equal(held[:, :2], had[:, :2]) and torch.equal(held[:, 2 + D:], had[:, 2 + D:]) and torch.equal(held[60:], had[60:])


def test_embedding_masked_rows_of_the_gradient(apex):
    """What stands at places without a token does not count, NaN included, and a NaN stays in its token's row."""
    N, V, D = 3000, 50, 20
    rng = np.random.default_rng(5)
    token = to_dev(rng.integers(-1, V, N).astype(np.int32))
    dout = to_dev(rng.standard_normal((N, D)).astype(np.float32))
    _, clean = apex.embedding_backward(dout, token, V)
    dout[token < 0] = NAN
    _, got = apex.embedding_backward(dout, token, V)
    assert torch.equal(got["dtable"], clean["dtable"])
    dout[(token == 7).nonzero()[0]] = NAN
    _, got = apex.embedding_backward(dout, token, V)
    assert got["dtable"][7].isnan().all()
    rows = [v for v in range(V) if v != 7]
    assert torch.equal(got["dtable"][rows], clean["dtable"][rows])


def test_embedding_same_bits_whatever_the_workspace_held(apex):
    for N, V in ((500, 300), (30000, 5000)):
        rng = np.random.default_rng(N)
        dout = to_dev(rng.standard_normal((N, 30)).astype(np.float32))
        space = apex.embedding_backward_workspace(N, V, 30)
        tokens = [to_dev(rng.integers(0, V, N).astype(np.int32)) for _ in range(2)]
        first = [apex.embedding_backward(dout, t, V)[1]["dtable"] for t in tokens]
        for _ in range(2):
            for t, f in zip(tokens, first):           # the other tokens' places are in the workspace
                rc, out = apex.embedding_backward(dout, t, V, workspace=space)
                assert rc == apex.OK and torch.equal(out["dtable"], f)


# --------------------------------------------------------------------------------------------------------- clipping

def clip_check(apex, grads, max_norm, **k):
    norm, want = plain.clip([plain.f64(x) for x in grads], max_norm)
    rc, out = apex.clip_gradients(grads, max_norm, **k)
    assert rc == apex.OK
    got = float(out["norm"])
    with np.errstate(over="ignore"):                               # (beyond the range of 32 bits the norm reads +inf)
        assert got == np.float32(norm) or abs(got - norm) <= norm * 2.0 ** -23
    for x, w, g in zip(out["out"], want, grads):
        check(x, w, abs(w) * 2.0 ** -22, g.dtype, "out")          # (the factor's rounding, twice, and the product's)
    return out


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("sizes", [(1,), (7, 0, 3), (8192,), (8191, 8193, 1), (100000, 5, 33333), tuple(range(250))], ids=lambda s: str(len(s)) + "x" + str(s[-1]))
def test_clipping(apex, dtype, sizes):
    rng = np.random.default_rng(len(sizes))
    grads = [to_dev(rng.standard_normal(n), DTYPES[dtype]) for n in sizes]
    n = sum(sizes)
    for max_norm in (0.5 * n ** 0.5, 2.0 * n ** 0.5):
        clip_check(apex, grads, max_norm, out=[torch.empty_like(x) for x in grads])
    had = [x.clone() for x in grads]
    want = apex.clip_gradients(grads, 0.25, out=[torch.empty_like(x) for x in grads])[1]
    rc, out = apex.clip_gradients(had, 0.25)
    assert rc == apex.OK and torch.equal(out["norm"], want["norm"])
    assert all(a is b for a, b in zip(out["out"], had)) and all(torch.equal(a, b) for a, b in zip(had, want["out"]))


def test_clipping_of_types_side_by_side_and_odd_addresses(apex):
    rng = np.random.default_rng(0)
    grads = [to_dev(rng.standard_normal((30, 41)), t) for t in DTYPES.values()] + [to_dev(rng.standard_normal(20000), torch.bfloat16)[3:]]
    clip_check(apex, grads, 7.0, out=[torch.empty_like(x) for x in grads])
    turned = to_dev(rng.standard_normal((30, 41)).astype(np.float32)).t()
    clip_check(apex, [turned], 1.0, out=[torch.empty_like(turned)])


def test_clipping_of_numbers_that_are_large_small_or_none(apex):
    ones = torch.ones(1000, device="cuda:0")
    big = clip_check(apex, [ones * 1e38, -ones], 1.0, out=[torch.empty_like(ones) for _ in range(2)])        # squares beyond 32 bits
    assert float(big["out"][0].abs().max()) > 0
    small = [ones * 1e-30]
    out = clip_check(apex, small, 1.0, out=[torch.empty_like(ones)])
    assert torch.equal(out["out"][0], small[0])
    zero = clip_check(apex, [ones * 0], 1.0, out=[torch.empty_like(ones)])
    assert float(zero["norm"]) == 0
    for bad in (NAN, float("inf"), -float("inf")):
        grads = [ones.clone(), ones.clone() * 50]
        grads[1][77] = bad
        had = [x.clone() for x in grads]
        for out in (None, [torch.empty_like(x) for x in grads]):
            rc, got = apex.clip_gradients(grads, 1.0, out=out)
            assert rc == apex.OK and not torch.isfinite(got["norm"]).any()
            for a, b in zip(got["out"], had):
                assert torch.equal(a.nan_to_num(123.0), b.nan_to_num(123.0))
    rc, got = apex.clip_gradients([ones], float("inf"))
    assert rc == apex.OK and abs(float(got["norm"]) - 1000 ** 0.5) < 1e-5 and (ones == 1).all()
    for none in ([], [torch.empty(0, device="cuda:0")]):
        rc, got = apex.clip_gradients(none, 1.0)
        assert rc == apex.OK and float(got["norm"]) == 0
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------------------------- streams and graphs

class Together:
    """A learner's step: tokens' rows, the delta rule over them and its gradient, the table's gradient, all of them clipped."""

    def __init__(self, apex, seed=0, S=3, T=100, V=50, H=2, D=32):
        self.apex, self.S, self.T, self.V = apex, S, T, V
        g = torch.Generator("cuda:0")
        g.manual_seed(seed)
        self.gen = g
        self.table = torch.randn((V, 3 * H * D), generator=g, device="cuda:0") / D ** 0.5
        self.token = torch.zeros((S * T,), dtype=torch.int32, device="cuda:0")
        self.gate = -torch.rand((S, T, H), generator=g, device="cuda:0")
        self.beta = torch.rand((S, T, H), generator=g, device="cuda:0")
        self.do = torch.randn((S, T, H, D), generator=g, device="cuda:0")
        self.h0 = torch.randn((S, H, D, D), generator=g, device="cuda:0")
        self.rows = torch.empty((S * T, 3 * H * D), device="cuda:0")
        parts = self.rows.view(S, T, 3, H, D).unbind(2)
        self.parts = parts
        self.drows = torch.empty_like(self.rows)
        self.out = dict(o=torch.empty_like(self.do), h_last=torch.empty_like(self.h0), carry=torch.empty(apex.delta_rule_carry_shape(S, T, H, D, D), device="cuda:0"))
        dparts = self.drows.view(S, T, 3, H, D).unbind(2)
        self.back = dict(zip(("dq", "dk", "dv"), dparts), dg=torch.empty_like(self.gate), dbeta=torch.empty_like(self.gate), dh0=torch.empty_like(self.h0))
        self.dtable = torch.empty_like(self.table)
        self.norm = torch.empty(1, device="cuda:0")
        self.spaces = [apex.delta_rule_workspace(S, T, H, D, D, backward=True), apex.embedding_backward_workspace(S * T, V, 3 * H * D),
                       apex.clip_gradients_workspace(3)]

    def refill(self):
        self.token.copy_(torch.randint(-1, self.V, self.token.shape, generator=self.gen, device="cuda:0", dtype=torch.int32))
        self.do.normal_(generator=self.gen)

    def run(self, stream=None):
        a, (q, k, v) = self.apex, self.parts
        assert a.embedding(self.table, self.token, out=dict(out=self.rows), stream=stream)[0] == a.OK
        more = dict(workspace=self.spaces[0], stream=stream)
        assert a.delta_rule(q, k, v, self.gate, self.beta, h0=self.h0, out=self.out, **more)[0] == a.OK
        assert a.delta_rule_backward(q, k, v, self.gate, self.beta, self.do, self.out["carry"], out=self.back, **more)[0] == a.OK
        assert a.embedding_backward(self.drows, self.token, self.V, out=dict(dtable=self.dtable), workspace=self.spaces[1], stream=stream)[0] == a.OK
        assert a.clip_gradients([self.dtable, self.back["dg"], self.back["dbeta"]], 1.0, norm=self.norm, workspace=self.spaces[2], stream=stream)[0] == a.OK

    def results(self):
        return [t.clone() for t in (self.rows, *self.out.values(), *self.back.values(), self.dtable, self.norm)]


def test_a_learning_step_of_them_together(apex):
    """Against the plain forms, one behind the other."""
    t = Together(apex)
    t.refill()
    t.run()
    torch.cuda.synchronize()
    token = t.token.cpu().numpy()
    rows = plain.embedding(plain.f64(t.table), token, 1.0)
    check(t.rows, rows, 0.0, torch.float32, "rows")
    q, k, v = (rows.reshape(t.S, t.T, 3, 2, 32)[:, :, i] for i in range(3))
    want = plain.delta(q, k, v, plain.f64(t.gate), plain.f64(t.beta), 1.0, None, None, plain.f64(t.h0), plain.f64(t.do), None)
    for n in ("dq", "dk", "dv", "dh0"):
        check(t.back[n], want[n], plain.delta_bound(n, want, 32, 32), torch.float32, n)
    drows = np.stack([want[n] for n in ("dq", "dk", "dv")], 2).reshape(t.S * t.T, -1)
    grads = [plain.embedding_backward(drows, token, t.V, 1.0)[0], want["dg"], want["dbeta"]]
    norm, clipped = plain.clip(grads, 1.0)
    assert abs(float(t.norm) - norm) < 1e-4 * norm
    for got, w in zip((t.dtable, t.back["dg"], t.back["dbeta"]), clipped):
        assert np.abs(plain.f64(got) - w).max() < 1e-4 * np.abs(w).max()


def test_learning_step_on_other_streams_and_in_a_graph(apex):
    t = Together(apex)
    t.refill()
    t.run()
    torch.cuda.synchronize()
    want = t.results()
    stream = torch.cuda.Stream()
    for x in (t.rows, t.drows, t.dtable, t.norm):
        x.fill_(NAN)
    stream.wait_stream(torch.cuda.current_stream())
    t.run(stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(t.results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.run()
    for _ in range(4):
        t.refill()
        t.run()
        torch.cuda.synchronize()
        want = t.results()
        for x in (t.rows, t.drows, t.dtable, t.norm):
            x.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(t.results(), want))


def test_calls_that_make_their_own_outputs_on_a_stream(apex):
    c = Delta(2, 90, 1, 2, 16, 24, "bf16", seed=2)
    want = c.run(apex)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = c.run(apex, stream=stream)
    for n in ("o", "h_last") + BACK:
        assert torch.equal(got[n], want[n]), n
    dout, token = torch.randn((300, 12), device="cuda:0"), torch.randint(0, 9, (300,), device="cuda:0", dtype=torch.int32)
    grads = [torch.randn(5000, device="cuda:0")]
    torch.cuda.synchronize()
    rows = apex.embedding(dout, token)[1]["out"], apex.embedding(dout, token, stream=stream)[1]["out"]
    back = apex.embedding_backward(dout, token, 9)[1]["dtable"], apex.embedding_backward(dout, token, 9, stream=stream)[1]["dtable"]
    norm = apex.clip_gradients(grads, float("inf"))[1]["norm"], apex.clip_gradients(grads, float("inf"), stream=stream)[1]["norm"]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in (rows, back, norm))


# --------------------------------------------------------------------------------------------------- refusals, sizes

def test_learning_operators_refuse_what_does_not_fit(apex):
    c = Delta(2, 100, 1, 2, 16, 24, "f32", seed=2)
    space = apex.delta_rule_workspace(2, 100, 2, 16, 24, backward=True)
    small = apex.delta_rule_workspace(2, 100, 2, 16, 24)
    rc, out = apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, carry=True, workspace=small)
    assert rc == apex.OK
    back = (c.q, c.k, c.v, c.g, c.beta, c.do, out["carry"])
    assert apex.delta_rule_backward(*back, workspace=space)[0] == apex.OK
    for call in (lambda: apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, workspace=small[:-1]), lambda: apex.delta_rule_backward(*back, workspace=small),
                 lambda: apex.delta_rule_backward(*back, workspace=space[:-1])):
        with pytest.raises(AssertionError, match="workspace"):
            call()
    half = c.q.half()
    for match, call in (("one floating type", lambda: apex.delta_rule(half, c.k, c.v, c.g, c.beta)),
                        ("q and k", lambda: apex.delta_rule(c.q, c.k[:, :50], c.v, c.g, c.beta)),
                        ("heads", lambda: apex.delta_rule(c.q, c.k, c.v.transpose(2, 3).contiguous().transpose(2, 3), c.g, c.beta)),
                        ("heads", lambda: apex.delta_rule(c.q[:, :, 0], c.k, c.v, c.g, c.beta, out=out, workspace=space)),
                        ("g:", lambda: apex.delta_rule(c.q, c.k, c.v, c.g[:, :50].contiguous(), c.beta)),
                        ("fp32", lambda: apex.delta_rule(c.q, c.k, c.v, c.g.half(), c.beta)),
                        ("h0", lambda: apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, h0=c.h0[:1])),
                        ("h0", lambda: apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, h0=torch.empty(0, device="cuda:0"))),
                        ("length", lambda: apex.delta_rule(c.q, c.k, c.v, c.g, c.beta, length=torch.zeros(3, dtype=torch.int32, device="cuda:0"))),
                        ("carry", lambda: apex.delta_rule_backward(c.q, c.k, c.v, c.g, c.beta, c.do, out["carry"][:, :1].contiguous())),
                        ("do", lambda: apex.delta_rule_backward(c.q, c.k, c.v, c.g, c.beta, c.do[:, :9], out["carry"])),
                        ("carry", lambda: apex.delta_rule_backward(c.q, c.k, c.v, c.g, c.beta, c.do, None))):
        with pytest.raises(AssertionError, match=match):
            call()
    assert apex.delta_rule(c.q[:, :, [0, 0, 0]], c.k[:, :, [0, 0, 0]], c.v, c.g, c.beta)[0] == apex.ERR_INVALID_ARG     # 2 heads over 3
    table, token = torch.zeros((9, 4), device="cuda:0"), torch.zeros(5, dtype=torch.int32, device="cuda:0")
    dout = torch.zeros((5, 4), device="cuda:0")
    space = apex.embedding_backward_workspace(5, 9, 4)
    for match, call in (("token", lambda: apex.embedding(table, token.long())), ("out", lambda: apex.embedding(table, token, out=dict(out=dout[:4]))),
                        ("table", lambda: apex.embedding(table.t(), token)), ("dout", lambda: apex.embedding_backward(dout[:4], token, 9)),
                        ("workspace", lambda: apex.embedding_backward(dout, token, 9, workspace=space[:256])),
                        ("dout", lambda: apex.embedding_backward(dout.half(), token, 9, out=dict(dtable=table))),
                        ("out", lambda: apex.clip_gradients([table], 1.0, out=[table.half()])), ("out", lambda: apex.clip_gradients([table], 1.0, out=[])),
                        ("dense", lambda: apex.clip_gradients([table[:, :2]], 1.0)), ("one device", lambda: apex.clip_gradients([table, table.cpu()], 1.0)), ("floating", lambda: apex.clip_gradients([token], 1.0)),
                        ("norm", lambda: apex.clip_gradients([table], 1.0, norm=torch.zeros(2, device="cuda:0"))),
                        ("workspace", lambda: apex.clip_gradients([table], 1.0, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda:0")))):
        with pytest.raises(AssertionError, match=match):
            call()
    assert apex.clip_gradients([table], 0.0)[0] == apex.ERR_INVALID_ARG
    torch.cuda.synchronize()


def test_rows_whose_offsets_pass_32_bits(apex):
    """Sequences, rows and tables whose elements lie beyond 2^32."""
    far = torch.empty((2, (1 << 32) + 4096), dtype=torch.bfloat16, device="cuda:0")
    S, T, H, D = 2, 70, 1, 16
    c = Delta(S, T, H, H, D, D, "bf16", seed=1)
    want = c.want()
    views = []
    for i, x in enumerate((c.q, c.k, c.v)):
        v = far.as_strided((S, T, H, D), (far.stride(0), D, D, 1), i * T * D)
        v.copy_(x)
        views.append(v)
    back = dict(dg=torch.empty_like(c.g), dbeta=torch.empty_like(c.g), dh0=torch.empty_like(c.h0))
    for i, n in enumerate(("dq", "dk", "dv")):
        back[n] = far.as_strided((S, T, H, D), (far.stride(0), D, D, 1), (i + 4) * T * D)
    c.check(c.run(apex, q=views[0], k=views[1], v=views[2], back=back), want)
    V, D = 5, 8
    table = far.view(-1).as_strided((V, D), (1 << 30, 1))
    table.copy_(torch.randn((V, D), device="cuda:0"))
    token = torch.tensor([4, 0, 4, 3], dtype=torch.int32, device="cuda:0")
    assert torch.equal(apex.embedding(table, token)[1]["out"], table[token.long()])
    dout = torch.randn((4, D), device="cuda:0").bfloat16()
    rc, _ = apex.embedding_backward(dout, token, V, out=dict(dtable=table))
    assert rc == apex.OK
    want, err = plain.embedding_backward(plain.f64(dout), token.cpu().numpy(), V, 1.0)
    check(table, want, err, torch.bfloat16, "dtable")
