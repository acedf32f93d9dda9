"""What a learner's step of a recurrent draft model needs between its tokens and its update, as measurable cases.

The draft looks its tokens up, carries a matrix per head from token to token by the gated delta rule, and is trained on what
the replay memory holds; its gradients are clipped by their norm over all of them before they are applied.

``delta``  the gated delta rule, over whole sequences with its gradient (learner) or without (prefill), and for single tokens
           (actor)
``embed``  the lookup of tokens' rows, scaled, and the gradient of the table
``clip``   the norm over many tensors, and the tensors scaled so that it stays below a limit

``own`` chooses between the plain forms below (elementary operations in 32 bits, rounded once at the end) and the calls of
``paper_1803_00933_amd.apex``.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GAMMA = 0.997
CHUNK = 64          # steps that the plain form of the delta rule takes at once
MAX_NORM = 40.0


def _delta(name, S, T, Hk, H, Dk, Dv, dtype, back, resets=False, ragged=False, joined=False):
    c = dict(op="delta", S=S, T=T, Hk=Hk, H=H, Dk=Dk, Dv=Dv, dtype=dtype, back=back, resets=resets, ragged=ragged, joined=joined)
    return dict(c, name=name) if name else c


def _embed(name, N, V, D, dtype, back, scaled=True, skewed=True, padded=False):
    c = dict(op="embed", N=N, V=V, D=D, dtype=dtype, back=back, scaled=scaled, skewed=skewed, padded=padded)
    return dict(c, name=name) if name else c


def _clip(name, V, D, layers, dtype, size):
    c = dict(op="clip", V=V, D=D, layers=layers, dtype=dtype, size=size)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token for each of 64 actors' sequences: the smallest call of the draft, bound by its states
        _delta("delta_step", 64, 1, 16, 16, 128, 128, "bf16", False),
        # a learner's batch of short replayed sequences of uneven lengths, which episodes' ends cut
        _delta("delta_replayed", 64, 96, 4, 8, 64, 64, "bf16", True, resets=True, ragged=True),
        # long sequences, queries, keys and values as the parts of one projection: the largest training call
        _delta("delta_long", 4, 8192, 8, 16, 128, 128, "bf16", True, joined=True),
        # odd sizes in 32 bits
        _delta("delta_odd", 3, 1501, 5, 5, 72, 100, "f32", True, resets=True),
        # one long prompt is read in: few heads, so there is little to share out but the columns of a state
        _delta("delta_prompt", 1, 16384, 8, 8, 128, 128, "f16", False),
        # an actor's tokens: latency
        _embed("embed_step", 64, 32000, 1024, "bf16", False),
        # a learner's batch of replayed sequences, padded where they are shorter, with the table's gradient
        _embed("embed_batch", 6144, 32768, 1024, "bf16", True, padded=True),
        # odd sizes in 32 bits, every token as likely as any other
        _embed("embed_odd", 7777, 49999, 1003, "f32", True, skewed=False),
        # long sequences and a large vocabulary: the largest
        _embed("embed_large", 32768, 131072, 2048, "bf16", True),
        # the gradients of a small draft: latency
        _clip("clip_small", 4096, 128, 1, "f32", 1.0),
        # an ordinary draft's gradients, whose norm is below the limit
        _clip("clip_draft", 32768, 1024, 4, "bf16", 1e-4),
        # many tensors of odd sizes
        _clip("clip_large", 131071, 2047, 10, "bf16", 0.01),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("delta", "delta", "embed", "clip"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op == "delta":
        S, T, Hk, share = _log(rng, 1, 128), _log(rng, 1, 16384), _log(rng, 1, 16), rng.choice((1, 1, 2, 3))
        Dk, Dv = (rng.choice((64, 128, rng.randint(8, 128))) for _ in range(2))
        T = max(1, min(T, 4 * 8192 * 16 * 128 * 128 // (S * Hk * share * 128 * 128 * (1 if dtype == "bf16" else 4))))
        return _delta(None, S, T, Hk, Hk * share, Dk, Dv, dtype, rng.random() < 0.6, resets=rng.random() < 0.5,
                      ragged=rng.random() < 0.5, joined=rng.random() < 0.5)
    if op == "embed":
        N, V, D = _log(rng, 1, 32768), _log(rng, 100, 131072), _log(rng, 16, 2048)
        if dtype == "f32":
            N, V = max(1, N // 2), max(100, V // 2)
        return _embed(None, N, V, D, dtype, rng.random() < 0.7, scaled=rng.random() < 0.5, skewed=rng.random() < 0.5,
                      padded=rng.random() < 0.5)
    return _clip(None, _log(rng, 100, 65536), _log(rng, 16, 2048), _log(rng, 1, 10), dtype, rng.choice((1e-4, 0.01, 1.0)))


# ---------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(DEVICE)
    g.manual_seed(seed)
    s = dict(case=case, **{"delta": _prepare_delta, "embed": _prepare_embed, "clip": _prepare_clip}[case["op"]](case, g))
    if own:
        s["kept"] = _kept(case, s)
    return s


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEVICE)


def _prepare_delta(c, g):
    """Queries and keys of unit length, values of unit size, decays that remember some tens to hundreds of steps, a stored
    start state."""
    S, T, Hk, H, Dk, Dv, dt = c["S"], c["T"], c["Hk"], c["H"], c["Dk"], c["Dv"], DTYPES[c["dtype"]]
    widths = (Hk * Dk, Hk * Dk, H * Dv)
    if c["joined"]:
        parts = torch.empty((S, T, sum(widths)), dtype=dt, device=DEVICE).split(widths, 2)
    else:
        parts = [torch.empty((S, T, w), dtype=dt, device=DEVICE) for w in widths]
    q, k, v = (p.unflatten(2, n) for p, n in zip(parts, ((Hk, Dk), (Hk, Dk), (H, Dv))))
    for i in range(S):
        for p in (q, k):
            x = _randn(g, T, Hk, Dk)
            p[i] = x / x.square().sum(2, keepdim=True).sqrt()
        v[i] = _randn(g, T, H, Dv)
    s = dict(q=q, k=k, v=v, g=-torch.exp(_randn(g, S, T, H) * 0.7 - 3.5), beta=torch.sigmoid(_randn(g, S, T, H)),
             h0=_randn(g, S, H, Dk, Dv) * 0.3, discount=None, length=None, scale=Dk ** -0.5)
    if c["resets"]:
        s["discount"] = (_rand(g, S, T) > 0.02).float() * GAMMA
    if c["ragged"]:
        s["length"] = torch.randint(0, T + 1, (S,), generator=g, device=DEVICE, dtype=torch.int32)
        s["length"][0] = T
    if c["back"]:
        s["do"], s["dh_last"] = _randn(g, S, T, H, Dv).to(dt), _randn(g, S, H, Dk, Dv) * 0.1
    return s


def _prepare_embed(c, g):
    """Tokens as frequent as one over their rank, or all alike; padded places hold -1."""
    N, V, D, dt = c["N"], c["V"], c["D"], DTYPES[c["dtype"]]
    table = torch.empty((V, D), dtype=dt, device=DEVICE)
    for i in range(0, V, 16384):
        table[i:i + 16384] = _randn(g, min(16384, V - i), D)
    u = _rand(g, N).double()
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0 if c["skewed"] else u * V).long().clamp(max=V - 1)
    token = torch.randperm(V, generator=g, device=DEVICE)[rank].int()
    if c["padded"]:
        token = torch.where(_rand(g, N) < 0.2, -1, token)
    s = dict(table=table, token=token, scale=D ** 0.5 if c["scaled"] else 1.0)
    if c["back"]:
        s["dout"] = _randn(g, N, D).to(dt)
    return s


def _prepare_clip(c, g):
    """The gradients of a table, of each layer's projections and of its vectors."""
    V, D = c["V"], c["D"]
    shapes = [(V, D)] + [s for _ in range(c["layers"]) for s in ((D, 2 * D), (D, D), (D, 4 * D), (4 * D, D), (D,), (D,))] + [(D,)]
    grads = []
    for shape in shapes:
        t = torch.empty(shape, dtype=DTYPES[c["dtype"]], device=DEVICE)
        flat = t.view(-1)
        for i in range(0, flat.numel(), 1 << 26):
            flat[i:i + (1 << 26)] = _randn(g, min(1 << 26, flat.numel() - i)) * c["size"]
        grads.append(t)
    return dict(grads=grads)


def _kept(c, s):
    """The workspace and the output buffers that a program keeps from call to call."""
    from paper_1803_00933_amd import apex
    if c["op"] == "clip":
        return dict(out=[torch.empty_like(t) for t in s["grads"]], norm=torch.empty(1, device=DEVICE),
                    workspace=apex.clip_gradients_workspace(s["grads"]))
    dt = DTYPES[c["dtype"]]
    if c["op"] == "embed":
        back = None
        if c["back"]:
            back = dict(out=dict(dtable=torch.empty((c["V"], c["D"]), dtype=dt, device=DEVICE)),
                        workspace=apex.embedding_backward_workspace(c["N"], c["V"], c["D"], device=DEVICE))
        return dict(out=dict(out=torch.empty((c["N"], c["D"]), dtype=dt, device=DEVICE)), back=back)
    S, T, H, Dk, Dv = c["S"], c["T"], c["H"], c["Dk"], c["Dv"]
    out = dict(o=torch.empty((S, T, H, Dv), dtype=dt, device=DEVICE), h_last=torch.empty((S, H, Dk, Dv), device=DEVICE))
    back = None
    if c["back"]:
        out["carry"] = torch.empty(apex.delta_rule_carry_shape(S, T, H, Dk, Dv), device=DEVICE)
        back = {"d" + n: torch.empty_strided(s[n].size(), s[n].stride(), dtype=dt, device=DEVICE) for n in ("q", "k", "v")}
        back.update(dg=torch.empty((S, T, H), device=DEVICE), dbeta=torch.empty((S, T, H), device=DEVICE),
                    dh0=torch.empty((S, H, Dk, Dv), device=DEVICE))
    return dict(out=out, back=back, workspace=apex.delta_rule_workspace(S, T, H, Dk, Dv, backward=c["back"], device=DEVICE))


# ------------------------------------------------------------------------------------------------------------- runs

def run(state):
    if own:
        return _run_own(state["case"], state)
    return {"delta": _plain_delta, "embed": _plain_embed, "clip": _plain_clip}[state["case"]["op"]](state["case"], state)


def _run_own(c, s):
    from paper_1803_00933_amd import apex
    kept = s["kept"]
    if c["op"] == "delta":
        more = dict(discount=s["discount"], length=s["length"], scale=s["scale"], workspace=kept["workspace"])
        rc, out = apex.delta_rule(s["q"], s["k"], s["v"], s["g"], s["beta"], h0=s["h0"], out=kept["out"], **more)
        assert rc == apex.OK
        got = dict(o=out["o"], h_last=out["h_last"])
        if c["back"]:
            rc, back = apex.delta_rule_backward(s["q"], s["k"], s["v"], s["g"], s["beta"], s["do"], out["carry"],
                                                dh_last=s["dh_last"], out=kept["back"], **more)
            assert rc == apex.OK
            got.update(back)
        return got
    if c["op"] == "embed":
        rc, out = apex.embedding(s["table"], s["token"], scale=s["scale"], out=kept["out"])
        assert rc == apex.OK
        got = dict(out)
        if c["back"]:
            rc, back = apex.embedding_backward(s["dout"], s["token"], c["V"], scale=s["scale"], **kept["back"])
            assert rc == apex.OK
            got.update(back)
        return got
    rc, out = apex.clip_gradients(s["grads"], MAX_NORM, out=kept["out"], norm=kept["norm"], workspace=kept["workspace"])
    assert rc == apex.OK
    return out


def _chunks(x, T, Tp):
    """[S,T,H,...] as [S,H,chunks,CHUNK,...], zeros behind the last step."""
    x = torch.cat((x, x.new_zeros((x.shape[0], Tp - T) + x.shape[2:])), 1).transpose(1, 2)
    return x.reshape(x.shape[:2] + (Tp // CHUNK, CHUNK) + x.shape[3:])


def _steps(x, T):
    """The other way round."""
    return x.flatten(2, 3)[:, :, :T].transpose(1, 2)


def _plain_delta(c, s):
    """Chunk by chunk: within one the steps' corrections are the solution of a triangular system, from one to the next goes
    the state."""
    S, T, Hk, H, Dk, Dv, dt, scale = c["S"], c["T"], c["Hk"], c["H"], c["Dk"], c["Dv"], DTYPES[c["dtype"]], s["scale"]
    Tp, share = -(-T // CHUNK) * CHUNK, c["H"] // c["Hk"]
    length = torch.full((S,), T, device=DEVICE) if s["length"] is None else s["length"].long()
    inside = torch.arange(T, device=DEVICE) < length[:, None]
    keep = torch.ones((S, T), device=DEVICE) if s["discount"] is None else (s["discount"] != 0).float()
    cut = torch.cat((torch.zeros((S, 1), device=DEVICE), 1.0 - keep[:, :-1]), 1) * inside
    masked = [torch.where(inside[:, :, None], x, 0.0) for x in (s["g"], s["beta"])]
    wide = [torch.where(inside[:, :, None, None], s[n].float(), 0.0) for n in ("q", "k", "v")]
    q, k = (_chunks(x.repeat_interleave(share, 2), T, Tp) for x in wide[:2])
    v = _chunks(wide[2], T, Tp)
    b = _chunks(masked[1], T, Tp)[..., None]
    G = _chunks(masked[0], T, Tp).double().cumsum(3)
    part = _chunks(cut[:, :, None], T, Tp).cumsum(3)                        # [S,1,chunks,CHUNK]
    place = torch.arange(CHUNK, device=DEVICE)
    before = place[:, None] > place
    D = torch.exp((G[..., :, None] - G[..., None, :]).float())
    D = torch.where((part[..., :, None] == part[..., None, :]) & (place[:, None] >= place), D, 0.0)
    gam = torch.where(part == 0, torch.exp(G.float()), 0.0)[..., None]      # what is left of the chunk's start state
    Gam = D[..., -1, :, None]                                               # what is left of a step at the chunk's end
    L = torch.where(before, k @ k.transpose(3, 4) * D, 0.0)
    M = L.clone()                                                           # M = L - L b M, row by row
    for t in range(1, CHUNK):
        M[..., t, :] -= ((L[..., t:t + 1, :t] * b[..., None, :t, 0]) @ M[..., :t, :])[..., 0, :]
    P = q @ k.transpose(3, 4) * D
    n = Tp // CHUNK
    kt, state, starts, E = k.transpose(3, 4), s["h0"], [], []
    for i in range(n):
        starts.append(state)
        X = v[:, :, i] - gam[:, :, i] * (k[:, :, i] @ state)
        E.append(X - M[:, :, i] @ (b[:, :, i] * X))
        state = gam[:, :, i, -1:] * state + kt[:, :, i] @ (Gam[:, :, i] * (b[:, :, i] * E[-1]))
    S0, E = torch.stack(starts, 2), torch.stack(E, 2)
    U = b * E
    o = scale * (gam * (q @ S0) + P @ U)
    rows, last = torch.arange(S, device=DEVICE), (length - 1).clamp(min=0)
    keep_last = torch.where(length > 0, keep[rows, last], 1.0)[:, None, None, None]
    out = dict(o=torch.where(inside[:, :, None, None], _steps(o, T), 0.0).to(dt), h_last=keep_last * state)
    if not c["back"]:
        return out
    do = _chunks(torch.where(inside[:, :, None, None], s["do"].float(), 0.0), T, Tp) * scale
    from_o, q_do = P.transpose(3, 4) @ do, q.transpose(3, 4) @ (gam * do)
    d_state, ends, Y = keep_last * s["dh_last"], [None] * n, [None] * n
    for i in reversed(range(n)):
        ends[i] = d_state
        dU = from_o[:, :, i] + Gam[:, :, i] * (k[:, :, i] @ d_state)
        Y[i] = dU - M[:, :, i].transpose(2, 3) @ (b[:, :, i] * dU)
        d_state = q_do[:, :, i] + gam[:, :, i, -1:] * d_state - kt[:, :, i] @ (gam[:, :, i] * b[:, :, i] * Y[i])
    dS, Y = torch.stack(ends, 2), torch.stack(Y, 2)
    dv = b * Y
    B1 = do @ U.transpose(3, 4) * D
    B2 = torch.where(before, dv @ U.transpose(3, 4) * D, 0.0)
    S0t, dSt = S0.transpose(3, 4), dS.transpose(3, 4)
    dq = gam * (do @ S0t) + B1 @ k
    U_end = Gam * U
    dk = U_end @ dSt + B1.transpose(3, 4) @ q - gam * (dv @ S0t) - B2 @ k - B2.transpose(3, 4) @ k
    dG = (q * dq).sum(4) - (v * dv).sum(4)
    at_end = (dS * (gam[:, :, :, -1:] * S0 + kt @ U_end)).sum((3, 4))
    same = (part[..., :, None] == part[..., None, :]) & (place[:, None] <= place)
    dg = torch.where(same, dG[..., None, :], 0.0).sum(4) + torch.where(part == part[..., -1:], at_end[..., None], 0.0)
    dg = torch.where(_chunks(cut[:, :, None], T, Tp) != 0, 0.0, dg)
    dq, dk = (_steps(x, T).unflatten(2, (Hk, share)).sum(3) for x in (dq, dk))
    out.update({n: torch.where(inside[:, :, None, None], x, 0.0).to(dt) for n, x in (("dq", dq), ("dk", dk), ("dv", _steps(dv, T)))})
    out.update(dg=torch.where(inside[:, :, None], _steps(dg, T), 0.0),
               dbeta=torch.where(inside[:, :, None], _steps((Y * E).sum(4), T), 0.0), dh0=d_state)
    return out


def _plain_embed(c, s):
    token = s["token"].long()
    named = (token >= 0)[:, None]
    row = token.clamp(min=0)
    out = dict(out=torch.where(named, s["table"][row].float() * s["scale"], 0.0).to(DTYPES[c["dtype"]]))
    if c["back"]:
        sums = torch.zeros((c["V"], c["D"]), device=DEVICE)
        sums.index_add_(0, row, torch.where(named, s["dout"].float(), 0.0))
        out["dtable"] = (sums * s["scale"]).to(DTYPES[c["dtype"]])
    return out


def _plain_clip(c, s):
    total = torch.zeros(1, dtype=torch.float64, device=DEVICE)
    for t in s["grads"]:
        total += t.float().square().sum(dtype=torch.float64)
    norm = total.sqrt()
    factor = (MAX_NORM / norm).clamp(max=1.0).float()
    return dict(norm=norm.float(), out=[(t.float() * factor).to(t.dtype) for t in s["grads"]])


# ------------------------------------------------------------------------------------------------- work and exactness

def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["op"] == "delta":
        n = c["S"] * c["T"]
        if c["ragged"]:
            n = n // 2
        state = 4 * c["S"] * c["H"] * c["Dk"] * c["Dv"]
        wide, gates = e * n * (2 * c["Hk"] * c["Dk"] + c["H"] * c["Dv"]), 8 * n * c["H"]
        out = e * n * c["H"] * c["Dv"]
        forward, backward = wide + gates + out + 2 * state, 2 * (wide + gates) + out + 2 * state
        flops = 6 * n * c["H"] * c["Dk"] * c["Dv"]
        return dict(bytes=forward + (backward if c["back"] else 0), flops=flops * (3 if c["back"] else 1))
    if c["op"] == "embed":
        n, row = c["N"], c["D"] * e
        distinct = min(n, c["V"]) // (4 if c["skewed"] else 1)
        forward, backward = n * (row + 4) + distinct * row, n * (row + 4) + c["V"] * row
        return dict(bytes=forward + (backward if c["back"] else 0), flops=n * c["D"] * (2 if c["back"] else 1))
    n = c["V"] * c["D"] + c["layers"] * (11 * c["D"] ** 2 + 2 * c["D"]) + c["D"]
    return dict(bytes=2 * n * e + 4, flops=3 * n)


def exact(case, seed):
    s = prepare(case, seed)
    return {"delta": _exact_delta, "embed": _exact_embed, "clip": _exact_clip}[case["op"]](case, s)


def _exact_delta(c, s):
    """Step by step, as the recurrence is written, with every state kept for the way back."""
    S, T, Hk, H, Dk, Dv, scale = c["S"], c["T"], c["Hk"], c["H"], c["Dk"], c["Dv"], s["scale"]
    per_state = S * H * Dk * Dv * 8
    if T * (60e-6 + per_state * 20e-12) * (6 if c["back"] else 2) > 15 or (c["back"] and T * per_state > 16e9):
        return None
    share = H // Hk
    q, k = (s[n].double().repeat_interleave(share, 2) for n in ("q", "k"))
    v, beta = s["v"].double(), s["beta"].double()
    decay = torch.exp(s["g"].double())
    ends = torch.zeros((S, T), dtype=torch.bool, device=DEVICE) if s["discount"] is None else s["discount"] == 0
    length = torch.full((S,), T, device=DEVICE) if s["length"] is None else s["length"].long()
    zero = torch.zeros((), dtype=torch.float64, device=DEVICE)
    state, o, kept = s["h0"].double(), torch.zeros((S, T, H, Dv), dtype=torch.float64, device=DEVICE), []
    for t in range(T):
        on = (length > t)[:, None, None, None]
        if c["back"]:
            kept.append(state)
        left = state * decay[:, t, :, None, None]
        u = beta[:, t, :, None] * (v[:, t] - (left * k[:, t, :, :, None]).sum(2))
        new = left + k[:, t, :, :, None] * u[:, :, None, :]
        o[:, t] = torch.where(on[..., 0], scale * (new * q[:, t, :, :, None]).sum(2), zero)
        state = torch.where(on, torch.where(ends[:, t, None, None, None], zero, new), state)
    out = dict(o=o, h_last=state)
    if not c["back"]:
        return out
    do, lam = s["do"].double() * scale, s["dh_last"].double()
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dg, dbeta = torch.zeros_like(beta), torch.zeros_like(beta)
    for t in reversed(range(T)):
        on = (length > t)[:, None, None, None]
        left = kept[t] * decay[:, t, :, None, None]
        miss = v[:, t] - (left * k[:, t, :, :, None]).sum(2)
        u = beta[:, t, :, None] * miss
        new = left + k[:, t, :, :, None] * u[:, :, None, :]
        at = torch.where(ends[:, t, None, None, None], zero, lam) + q[:, t, :, :, None] * do[:, t, :, None, :]   # of the new state
        du = (at * k[:, t, :, :, None]).sum(2)
        dmiss = beta[:, t, :, None] * du
        dleft = at - k[:, t, :, :, None] * dmiss[:, :, None, :]
        for held, x in ((dq, (new * do[:, t, :, None, :]).sum(3)), (dv, dmiss),
                        (dk, (at * u[:, :, None, :]).sum(3) - (left * dmiss[:, :, None, :]).sum(3))):
            held[:, t] = torch.where(on[..., 0], x, zero)
        dbeta[:, t] = torch.where(on[..., 0, 0], (du * miss).sum(2), zero)
        dg[:, t] = torch.where(on[..., 0, 0], (dleft * left).sum((2, 3)), zero)
        lam = torch.where(on, dleft * decay[:, t, :, None, None], lam)
    dq, dk = (x.unflatten(2, (Hk, share)).sum(3) for x in (dq, dk))
    out.update(dq=dq, dk=dk, dv=dv, dg=dg, dbeta=dbeta, dh0=lam)
    return out


def _exact_embed(c, s):
    token = s["token"].long()
    at = (token >= 0).nonzero()[:, 0]
    out = torch.zeros((c["N"], c["D"]), dtype=torch.float64, device=DEVICE)
    out[at] = s["table"].double()[token[at]] * s["scale"]
    if not c["back"]:
        return dict(out=out)
    dtable = torch.zeros((c["V"], c["D"]), dtype=torch.float64, device=DEVICE)
    dtable.index_put_((token[at],), s["dout"].double()[at] * s["scale"], accumulate=True)
    return dict(out=out, dtable=dtable)


def _exact_clip(c, s):
    norm = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in s["grads"]))
    return dict(norm=torch.tensor([norm], dtype=torch.float64), out=[t.double() * min(1.0, MAX_NORM / norm) for t in s["grads"]])
