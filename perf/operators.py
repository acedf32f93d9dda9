"""The operators around the replay memory of a recurrent draft model, as measurable cases.

An actor drafts tokens with a small recurrent model and has them verified against the target's probabilities; what the
target answered goes into the replay memory; the learner runs the draft over the sampled sequences and distils the
target's top logits into it.  Three operators carry that:

``scan``     the gated linear recurrence, over whole sequences with its gradient (learner) or without (prefill), and for
             single tokens (actor)
``distill``  the loss against a teacher's top logits, with the gradient of the student's logits
``verify``   which drafted tokens stand, and the token that follows them

``own`` chooses between the plain forms below (elementary operations in 32 bits, rounded once at the end) and the calls of
``paper_1803_00933_amd.apex``.
"""
import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GAMMA = 0.997
ACCEPTED = 0.8      # share of drafted tokens that stand, about, with the noise that _prepare_verify puts on the logits
ONE = 1 << 40       # the integer mass of probability 1
LOW = (1 << 32) - 1


def _scan(name, S, T, D, dtype, gate, back, resets=False, ragged=False, halves=False):
    c = dict(op="scan", S=S, T=T, D=D, dtype=dtype, gate=gate, back=back, resets=resets, ragged=ragged, halves=halves)
    return dict(c, name=name) if name else c


def _distill(name, N, V, K, dtype, rest=False, temperature=1.0, weighted=True, pad=0):
    c = dict(op="distill", N=N, V=V, K=K, dtype=dtype, rest=rest, temperature=temperature, weighted=weighted, pad=pad)
    return dict(c, name=name) if name else c


def _verify(name, B, G, V, dtype, ragged=False):
    c = dict(op="verify", B=B, G=G, V=V, dtype=dtype, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token for each of 64 actors' sequences: the smallest call of the draft, where latency counts
        _scan("scan_step", 64, 1, 1024, "bf16", "sigmoid", False),
        # a learner's batch of short replayed sequences of uneven lengths, which episodes' ends cut
        _scan("scan_replayed", 64, 96, 1024, "bf16", "sigmoid", True, resets=True, ragged=True),
        # long sequences, with gate and input as the halves of one projection: the largest training call
        _scan("scan_long", 4, 8192, 2048, "bf16", "sigmoid", True, halves=True),
        # odd sizes in 32 bits, the gate given by the caller, forward alone
        _scan("scan_odd", 3, 5001, 1003, "f32", "given", False, resets=True),
        # one long prompt is read in: few channels, so the length has to be shared out
        _scan("scan_prompt", 1, 32768, 768, "f16", "sigmoid", False),
        # a few positions, in 32 bits: fewer rows than the chip has compute units
        _distill("distill_few", 12, 32000, 32, "f32"),
        # an ordinary learner's batch
        _distill("distill_batch", 2048, 32768, 64, "bf16"),
        # odd sizes in a padded vocabulary, softened
        _distill("distill_odd", 777, 49999, 17, "f16", temperature=2.0, pad=33),
        # a large vocabulary, with the mass outside the named tokens as a class of its own: the largest call
        _distill("distill_large", 3001, 131072, 128, "bf16", rest=True),
        # one sequence is served: latency
        _verify("verify_one", 1, 4, 131072, "f32"),
        # a serving batch of sequences whose drafts end at different lengths
        _verify("verify_batch", 64, 5, 32768, "bf16", ragged=True),
        # many sequences, an odd large vocabulary
        _verify("verify_large", 256, 6, 128001, "f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("scan", "distill", "verify"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op == "scan":
        S, T, D = _log(rng, 1, 256), _log(rng, 1, 32768), _log(rng, 16, 4096)
        T = max(1, min(T, 4 * 8192 * 2048 * 2 // (S * D * SIZE[dtype])))
        return _scan(None, S, T, D, dtype, rng.choice(("given", "sigmoid")), rng.random() < 0.6, resets=rng.random() < 0.5,
                     ragged=rng.random() < 0.5, halves=rng.random() < 0.5)
    if op == "distill":
        N, V = _log(rng, 1, 8192), _log(rng, 1000, 200000)
        N = max(1, min(N, 3001 * 131072 * 2 // (V * SIZE[dtype])))
        return _distill(None, N, V, _log(rng, 1, 256), dtype, rest=rng.random() < 0.5, temperature=rng.choice((1.0, 1.0, 1.5, 4.0)),
                        weighted=rng.random() < 0.7, pad=rng.choice((0, 0, 7, 64)))
    B, G, V = _log(rng, 1, 512), rng.randint(1, 8), _log(rng, 1000, 200000)
    B = max(1, min(B, 256 * 13 * 128001 * 4 // ((2 * G + 1) * V * SIZE[dtype])))
    return _verify(None, B, G, V, dtype, ragged=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(DEVICE)
    g.manual_seed(seed)
    s = dict(case=case, **{"scan": _prepare_scan, "distill": _prepare_distill, "verify": _prepare_verify}[case["op"]](case, g))
    if own:
        s["kept"] = _kept(case, s)
    return s


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _prepare_scan(c, g):
    """Projections' outputs: gates that keep most of a state, inputs of unit size; a stored start state."""
    S, T, D, dt = c["S"], c["T"], c["D"], DTYPES[c["dtype"]]
    both = torch.empty((S, T, 2 * D) if c["halves"] else (2, S, T, D), dtype=dt, device=DEVICE)
    gate, x = (both[:, :, :D], both[:, :, D:]) if c["halves"] else (both[0], both[1])
    for i in range(S):
        gate[i] = (_randn(g, T, D) * 1.5 + 2.0) if c["gate"] == "sigmoid" else 1.0 - torch.rand((T, D), generator=g, device=DEVICE) * 0.3
        x[i] = _randn(g, T, D)
    s = dict(gate=gate, x=x, h0=_randn(g, S, D) * 0.3, discount=None, length=None)
    if c["resets"]:
        s["discount"] = (torch.rand((S, T), generator=g, device=DEVICE) > 0.02).float() * GAMMA
    if c["ragged"]:
        s["length"] = torch.randint(0, T + 1, (S,), generator=g, device=DEVICE, dtype=torch.int32)
        s["length"][0] = T
    if c["back"]:
        s["dh"], s["dh_last"] = _randn(g, S, T, D).to(dt), _randn(g, S, D)
    return s


def _prepare_distill(c, g):
    """Logits of a student that is near its teacher, and the teacher's largest."""
    N, V, K, dt, tau = c["N"], c["V"], c["K"], DTYPES[c["dtype"]], c["temperature"]
    held = torch.zeros((N, V + c["pad"]), dtype=dt, device=DEVICE)
    index = torch.empty((N, K), dtype=torch.int32, device=DEVICE)
    value, lse = torch.empty((N, K), device=DEVICE), torch.empty(N, device=DEVICE)
    for i in range(0, N, 256):
        z = _randn(g, min(256, N - i), V) * 2.0
        held[i:i + 256, :V] = z
        z += _randn(g, *z.shape) * 0.7
        v, j = z.topk(K, dim=1)
        value[i:i + 256], index[i:i + 256], lse[i:i + 256] = v, j.int(), torch.logsumexp(z / tau, dim=1)
    weight = torch.rand(N, generator=g, device=DEVICE) * 0.9 + 0.1 if c["weighted"] else None
    return dict(logits=held[:, :V], index=index, value=value, top_lse=lse if c["rest"] else None, weight=weight)


def _prepare_verify(c, g):
    """Probabilities of a draft and of a target near it, tokens drawn from the draft's, uniform 64-bit integers."""
    B, G, V, dt = c["B"], c["G"], c["V"], DTYPES[c["dtype"]]
    target = torch.empty((B, G + 1, V), dtype=dt, device=DEVICE)
    draft = torch.empty((B, G, V), dtype=dt, device=DEVICE)
    token = torch.empty((B, G), dtype=torch.int32, device=DEVICE)
    for b in range(0, B, 32):
        z = _randn(g, min(32, B - b), G + 1, V) * 2.5
        target[b:b + 32] = torch.softmax(z + _randn(g, *z.shape) * 0.5, dim=2)
        q = torch.softmax(z[:, :G], dim=2)
        draft[b:b + 32] = q
        wait = torch.empty_like(q).exponential_(generator=g)
        token[b:b + 32] = (q / wait).argmax(dim=2).int()
    rnd = torch.randint(-(1 << 63), (1 << 63) - 1, (B, G + 1), generator=g, device=DEVICE, dtype=torch.int64)
    length = torch.randint(0, G + 1, (B,), generator=g, device=DEVICE, dtype=torch.int32) if c["ragged"] else None
    return dict(target=target, draft=draft, token=token, rnd=rnd, length=length)


def _kept(c, s):
    """The workspace and the output buffers that a program keeps from call to call."""
    from paper_1803_00933_amd import apex
    if c["op"] == "scan":
        S, T, D, dt = c["S"], c["T"], c["D"], DTYPES[c["dtype"]]
        out = dict(h=torch.empty((S, T, D), dtype=dt, device=DEVICE), h_last=torch.empty((S, D), device=DEVICE))
        back = None
        if c["back"]:
            out["carry"] = torch.empty(apex.gated_scan_carry_shape(S, T, D), device=DEVICE)
            back = dict(dg=torch.empty_strided(s["gate"].size(), s["gate"].stride(), dtype=dt, device=DEVICE),
                        dx=torch.empty_strided(s["x"].size(), s["x"].stride(), dtype=dt, device=DEVICE),
                        dh0=torch.empty((S, D), device=DEVICE))
        return dict(out=out, back=back, workspace=apex.gated_scan_workspace(S, T, D, device=DEVICE))
    if c["op"] == "distill":
        N = c["N"]
        grad = torch.empty((N, c["V"] + c["pad"]), dtype=DTYPES[c["dtype"]], device=DEVICE)[:, :c["V"]]
        return dict(out=dict(loss=torch.empty(N, device=DEVICE), lse=torch.empty(N, device=DEVICE), grad=grad),
                    workspace=apex.distill_topk_workspace(N, c["V"], device=DEVICE))
    out = dict(accepted=torch.empty(c["B"], dtype=torch.int32, device=DEVICE),
               token=torch.empty((c["B"], c["G"] + 1), dtype=torch.int32, device=DEVICE))
    return dict(out=out, workspace=apex.verify_draft_workspace(c["B"], c["V"], device=DEVICE))


# ------------------------------------------------------------------------------------------------------------- runs

def run(state):
    if own:
        return _run_own(state["case"], state)
    return {"scan": _plain_scan, "distill": _plain_distill, "verify": _plain_verify}[state["case"]["op"]](state["case"], state)


def _run_own(c, s):
    from paper_1803_00933_amd import apex
    k = s["kept"]
    if c["op"] == "scan":
        rc, out = apex.gated_scan(s["gate"], s["x"], gate=c["gate"], discount=s["discount"], length=s["length"], h0=s["h0"],
                                  out=k["out"], workspace=k["workspace"])
        assert rc == apex.OK
        got = dict(h=out["h"], h_last=out["h_last"])
        if c["back"]:
            rc, back = apex.gated_scan_backward(s["gate"], s["x"], s["dh"], out["carry"], gate=c["gate"], discount=s["discount"],
                                                length=s["length"], dh_last=s["dh_last"], out=k["back"], workspace=k["workspace"])
            assert rc == apex.OK
            got.update(back)
        return got
    if c["op"] == "distill":
        rc, out = apex.distill_topk(s["logits"], s["index"], s["value"], weight=s["weight"], top_lse=s["top_lse"],
                                    temperature=c["temperature"], out=k["out"], workspace=k["workspace"])
    else:
        rc, out = apex.verify_draft(s["target"], s["draft"], s["token"], s["rnd"], length=s["length"], out=k["out"],
                                    workspace=k["workspace"])
    assert rc == apex.OK
    return out


def _composed(a, b):
    """All prefixes of the composition of h -> a h + b along dimension 1, by doubling: log2 T passes."""
    d, T = 1, a.shape[1]
    while d < T:
        b = torch.cat((b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]), 1)
        a = torch.cat((a[:, :d], a[:, d:] * a[:, :-d]), 1)
        d *= 2
    return a, b


def _plain_scan(c, s):
    gate, x, h0, dt = s["gate"].float(), s["x"].float(), s["h0"], DTYPES[c["dtype"]]
    S, T, D = x.shape
    if c["gate"] == "sigmoid":
        a, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
        b = rest * x
    else:
        a, b = gate, x
    keep = torch.ones((S, T), device=DEVICE) if s["discount"] is None else (s["discount"] != 0).float()
    length = torch.full((S,), T, device=DEVICE) if s["length"] is None else s["length"].long()
    inside = (torch.arange(T, device=DEVICE) < length[:, None])[:, :, None]
    before = torch.cat((torch.ones((S, 1), device=DEVICE), keep[:, :-1]), 1)[:, :, None]      # k_{t-1}
    a = torch.where(inside, a, 0.0)
    b = torch.where(inside, b, 0.0)
    A, h = _composed(a * before, b)
    h = torch.where(inside, h + A * h0[:, None], 0.0)
    some = (length > 0)[:, None]
    last = (length - 1).clamp(min=0)
    rows = torch.arange(S, device=DEVICE)
    keep_last = keep[rows, last][:, None]
    out = dict(h=h.to(dt), h_last=torch.where(some, keep_last * h[rows, last], h0))
    if not c["back"]:
        return out
    dh = torch.where(inside, s["dh"].float(), 0.0)
    dh[rows, last] += torch.where(some, keep_last * s["dh_last"], 0.0)
    after = torch.cat(((a * before)[:, 1:], torch.zeros((S, 1, D), device=DEVICE)), 1)         # k_t a_{t+1}
    _, lam = _composed(after.flip(1), dh.flip(1))
    lam = lam.flip(1)
    prev = before * torch.cat((h0[:, None], h[:, :-1]), 1)
    if c["gate"] == "sigmoid":
        dg, dx = lam * (prev - x) * a * rest, lam * rest
    else:
        dg, dx = lam * prev, lam
    out.update(dg=torch.where(inside, dg, 0.0).to(dt), dx=torch.where(inside, dx, 0.0).to(dt),
               dh0=torch.where(some, a[:, 0] * lam[:, 0], s["dh_last"]))
    return out


def _plain_distill(c, s):
    tau, index = c["temperature"], s["index"].long()
    z, t = s["logits"].float() / tau, s["value"].float() / tau
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    p = e / total
    if s["top_lse"] is None:
        t_top = t.max(1, keepdim=True).values
        log_q = t - t_top - torch.log(torch.exp(t - t_top).sum(1, keepdim=True))
    else:
        log_q = t - s["top_lse"][:, None]
    q = torch.exp(log_q)
    loss = (q * (log_q - (z.gather(1, index) - lse))).sum(1)
    if s["top_lse"] is None:
        grad = p * q.sum(1, keepdim=True)
    else:
        mass = q.sum(1, keepdim=True)
        rest = (1.0 - mass).clamp(min=0.0)
        e = e.scatter(1, index, 0.0)
        others = e.sum(1, keepdim=True)
        log_s = torch.log(others) - torch.log(total)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - log_s), 0.0)[:, 0]
        grad = p * (mass + rest) - e * (rest / others)
    grad = grad.scatter_add(1, index, -q) / tau
    if s["weight"] is not None:
        grad = grad * s["weight"][:, None]
    return dict(loss=loss, lse=lse[:, 0], grad=grad.to(s["logits"].dtype))


def _high_product(u, m):
    """floor(u m / 2^64) of unsigned 64-bit u (held in int64) and 0 <= m < 2^61, by halves that stay within 63 bits."""
    uh, ul, mh, ml = (u >> 32) & LOW, u & LOW, m >> 31, m & 0x7fffffff
    a, b = ul * mh, ul * ml
    low = (a >> 1) + ((((a & 1) << 31) + b) >> 32)                # floor(ul m / 2^32)
    a, b = uh * mh, uh * ml
    e = ((a & 1) << 31) + b
    return (a >> 1) + (e >> 32) + (low >> 32) + (((e & LOW) + (low & LOW)) >> 32)


def _masses(x):
    x = x.float()
    return (torch.where(x > 0, x, 0.0).clamp(max=1.0) * float(ONE)).to(torch.int64)


def _plain_verify(c, s):
    B, G = s["token"].shape
    token, rows = s["token"].long(), torch.arange(B, device=DEVICE)
    length = torch.full((B,), G, device=DEVICE) if s["length"] is None else s["length"].long()
    mp = _masses(s["target"][:, :G].gather(2, token[:, :, None])[:, :, 0])
    mq = _masses(s["draft"].gather(2, token[:, :, None])[:, :, 0])
    place = torch.arange(G + 1, device=DEVICE)
    stands = (_high_product(s["rnd"][:, :G], mq) < mp) & (place[:G] < length[:, None])
    n = stands.long().cumprod(1).sum(1)
    p = _masses(s["target"][rows, n])
    q = torch.where((n < length)[:, None], _masses(s["draft"][rows, n.clamp(max=G - 1)]), 0)
    left = (p - q).clamp(min=0)
    left = torch.where(left.sum(1, keepdim=True) > 0, left, p)
    up_to = left.cumsum(1)
    x = _high_product(s["rnd"][:, G], up_to[:, -1])
    drawn = torch.where(up_to[:, -1] > 0, (up_to <= x[:, None]).sum(1), -1)
    drafted = torch.cat((token, torch.zeros((B, 1), dtype=torch.int64, device=DEVICE)), 1)
    out = torch.where(place < n[:, None], drafted, torch.where(place == n[:, None], drawn[:, None], -1))
    return dict(accepted=n.int(), token=out.int())


# ------------------------------------------------------------------------------------------------- work and exactness

def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["op"] == "scan":
        n, state = c["S"] * c["T"] * c["D"], 4 * c["S"] * c["D"]
        forward, backward = 3 * n * e + 2 * state, 5 * n * e + 2 * state
        return dict(bytes=forward + (backward if c["back"] else 0), flops=n * (16 if c["back"] else 6))
    if c["op"] == "distill":
        n = c["N"] * c["V"]
        return dict(bytes=2 * n * e + c["N"] * (8 * c["K"] + 12), flops=8 * n)
    drafted = c["G"] / 2 if c["ragged"] else c["G"]
    rows = c["B"] * (2 - ACCEPTED ** drafted)          # the target's row, and the draft's where a token was turned down
    return dict(bytes=rows * c["V"] * e + c["B"] * (c["G"] * 20 + 16), flops=3 * rows * c["V"])


def exact(case, seed):
    s = prepare(case, seed)
    return {"scan": _exact_scan, "distill": _exact_distill, "verify": _exact_verify}[case["op"]](case, s)


def _exact_scan(c, s):
    """Step by step, as the recurrence is written."""
    S, T, D = c["S"], c["T"], c["D"]
    if T * (2 if c["back"] else 1) > 40000:
        return None
    gate, x = s["gate"].double(), s["x"].double()
    a = 1 / (1 + torch.exp(-gate)) if c["gate"] == "sigmoid" else gate
    b = x / (1 + torch.exp(gate)) if c["gate"] == "sigmoid" else x
    length = torch.full((S, 1), T, device=DEVICE) if s["length"] is None else s["length"].long()[:, None]
    ends = torch.zeros((S, T), dtype=torch.bool, device=DEVICE) if s["discount"] is None else s["discount"] == 0
    zero = torch.zeros((), dtype=torch.float64, device=DEVICE)
    state, h, prev = s["h0"].double(), torch.zeros_like(x), torch.zeros_like(x)
    for t in range(T):
        inside = length > t
        prev[:, t] = state
        new = a[:, t] * state + b[:, t]
        h[:, t] = torch.where(inside, new, zero)
        state = torch.where(inside, torch.where(ends[:, t, None], zero, new), state)
    out = dict(h=h, h_last=state)
    if c["back"]:
        lam, dg, dx = s["dh_last"].double(), torch.zeros_like(x), torch.zeros_like(x)
        for t in reversed(range(T)):
            inside = length > t
            at = torch.where(ends[:, t, None], zero, lam) + s["dh"][:, t].double()
            da, db = at * prev[:, t], at
            if c["gate"] == "sigmoid":
                da, db = (da - db * x[:, t]) * a[:, t] / (1 + torch.exp(gate[:, t])), db / (1 + torch.exp(gate[:, t]))
            dg[:, t], dx[:, t] = torch.where(inside, da, zero), torch.where(inside, db, zero)
            lam = torch.where(inside, a[:, t] * at, lam)
        out.update(dg=dg, dx=dx, dh0=lam)
    return out


def _exact_distill(c, s):
    N, V, tau = c["N"], c["V"], c["temperature"]
    loss, lse = (torch.empty(N, dtype=torch.float64, device=DEVICE) for _ in range(2))
    grad = torch.empty((N, V), dtype=torch.float64, device=DEVICE)
    for i in range(0, N, 64):
        z, j = s["logits"][i:i + 64].double() / tau, s["index"][i:i + 64].long()
        t = s["value"][i:i + 64].double() / tau
        lse[i:i + 64] = torch.logsumexp(z, 1)
        log_p = z - lse[i:i + 64, None]
        named = torch.zeros_like(z, dtype=torch.bool).scatter_(1, j, True)
        log_q = t - (torch.logsumexp(t, 1) if s["top_lse"] is None else s["top_lse"][i:i + 64].double())[:, None]
        q = log_q.exp()
        l = (q * (log_q - log_p.gather(1, j))).sum(1)
        g = log_p.exp() * q.sum(1, keepdim=True) - torch.zeros_like(z).scatter_(1, j, q)
        if s["top_lse"] is not None:
            r = 1 - q.sum(1)
            others = log_p.masked_fill(named, -float("inf"))
            log_s = torch.logsumexp(others, 1)
            l = l + torch.where(r > 0, r * (r.clamp(min=1e-300).log() - log_s), 0.0)
            g = g + r.clamp(min=0)[:, None] * (log_p.exp() - (others - log_s[:, None]).exp())
        w = 1.0 if s["weight"] is None else s["weight"][i:i + 64, None].double()
        loss[i:i + 64], grad[i:i + 64] = l, g * w / tau
    return dict(loss=loss, lse=lse, grad=grad)


def _exact_verify(c, s):
    """Sequence by sequence, with whole numbers of any size."""
    B, G = c["B"], c["G"]

    def mass(row):
        return np.floor(np.clip(row.double().cpu().numpy(), 0.0, 1.0) * ONE).astype(np.int64)

    rnd, token = s["rnd"].cpu().numpy().view(np.uint64), s["token"].cpu().numpy()
    at = s["token"].long()[:, :, None]
    p_at, q_at = mass(s["target"][:, :G].gather(2, at)), mass(s["draft"].gather(2, at))
    length = [G] * B if s["length"] is None else s["length"].tolist()
    accepted, out = np.zeros(B, np.int32), np.full((B, G + 1), -1, np.int32)
    for b in range(B):
        n = 0
        while n < length[b] and (int(rnd[b, n]) * int(q_at[b, n, 0])) >> 64 < int(p_at[b, n, 0]):
            out[b, n] = token[b, n]
            n += 1
        m = p = mass(s["target"][b, n])
        if n < length[b]:
            m = np.maximum(p - mass(s["draft"][b, n]), 0)
            m = m if m.any() else p
        up_to = np.cumsum(m)
        if up_to[-1]:
            out[b, n] = np.searchsorted(up_to, (int(rnd[b, G]) * int(up_to[-1])) >> 64, side="right")
        accepted[b] = n
    return dict(accepted=torch.from_numpy(accepted), token=torch.from_numpy(out))
