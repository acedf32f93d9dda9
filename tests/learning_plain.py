"""Plain 64-bit forms of the operators of a draft's learning step (gated delta rule, embedding, clipped gradients), and what their
32-bit kernels may be off by.

The delta rule's bound: a step of the recurrence is a contraction for keys of unit length and strengths up to 2, so what a step adds
to the error stays as large as it was, and a piece of 64 steps adds what its sums of products add: at most n 2^-24 times the sum of
the terms' magnitudes, n the additions that a number goes through one after the other (Dk for K S, 64 for the substitution, 64 for M X,
64 for the steps' sum, Dv for the sums over columns; twice for the way back, which starts from what the way there left).  `mag` is
the sum of magnitudes of each output's last sum, its largest over a sequence and head: errors of the states and corrections are
relative to the largest of these."""
import numpy as np

PIECE = 64


def f64(t):
    return t.detach().double().cpu().numpy()


def delta(q, k, v, g, beta, scale, discount=None, length=None, h0=None, do=None, dh_last=None):
    """Step by step.  Returns outputs by name, and the largest magnitude per sequence and head [S,H] under name + "_mag"."""
    S, T, Hk, Dk = q.shape
    H, Dv = v.shape[2:]
    share = H // Hk
    q, k = np.repeat(q, share, 2), np.repeat(k, share, 2)
    h0 = np.zeros((S, H, Dk, Dv)) if h0 is None else h0
    length = np.full(S, T) if length is None else np.clip(length, 0, T)
    keep = np.ones((S, T), bool) if discount is None else discount != 0
    out = dict(o=np.zeros((S, T, H, Dv)), h_last=h0.copy(), carry=np.zeros((S, -(-T // PIECE), H, Dk, Dv)))
    mag = {n: np.zeros((S, H)) for n in ("o", "h_last", "dq", "dk", "dv", "dbeta", "dg", "dh0")}
    back = do is not None
    if back:
        out.update(dq=np.zeros(q.shape), dk=np.zeros(q.shape), dv=np.zeros(v.shape), dg=np.zeros((S, T, H)), dbeta=np.zeros((S, T, H)),
                   dh0=np.zeros(h0.shape) if dh_last is None else dh_last.copy())
    decay = np.exp(np.float64(g))
    decay = np.where(np.exp(np.float32(g)) == 0, 0.0, decay)     # whose exponential is 0 in 32 bits: a cut

    def largest(name, s, x):
        mag[name][s] = np.maximum(mag[name][s], x.reshape(H, -1).max(1))

    for s in range(S):
        state, lefts, states = h0[s], [], []
        for t in range(length[s]):
            if t % PIECE == 0:
                out["carry"][s, t // PIECE] = state
            cut = decay[s, t] == 0
            left = np.where(cut[:, None, None], 0.0, state * decay[s, t][:, None, None])
            miss = v[s, t] - np.einsum("hkv,hk->hv", left, k[s, t])
            u = beta[s, t][:, None] * miss
            new = left + k[s, t][:, :, None] * u[:, None]
            out["o"][s, t] = scale * np.einsum("hkv,hk->hv", new, q[s, t])
            largest("o", s, abs(scale) * np.einsum("hkv,hk->hv", abs(left) + abs(k[s, t][:, :, None] * u[:, None]), abs(q[s, t])))
            largest("h_last", s, abs(left) + abs(k[s, t][:, :, None] * u[:, None]))
            lefts.append(left), states.append(new)
            state = new if keep[s, t] else np.zeros_like(new)
        largest("h_last", s, abs(h0[s]))
        out["h_last"][s] = state
        if not back or length[s] == 0:
            continue
        lam = np.zeros((H, Dk, Dv)) if dh_last is None else dh_last[s]
        ends = 0.0
        for t in reversed(range(length[s])):
            left, new = lefts[t], states[t]
            lam = lam if keep[s, t] else np.zeros_like(lam)
            if t % PIECE == PIECE - 1 or t == length[s] - 1:
                ends = abs(lam * new).sum((1, 2))
                row_sums = np.zeros(H)
            miss = v[s, t] - np.einsum("hkv,hk->hv", left, k[s, t])
            u = beta[s, t][:, None] * miss
            d = do[s, t] * scale
            at = lam + q[s, t][:, :, None] * d[:, None]
            du = np.einsum("hkv,hk->hv", at, k[s, t])
            dmiss = beta[s, t][:, None] * du
            cut = decay[s, t] == 0
            dleft = np.where(cut[:, None, None], 0.0, at - k[s, t][:, :, None] * dmiss[:, None])
            dq, dk = np.einsum("hkv,hv->hk", new, d), np.einsum("hkv,hv->hk", at, u) - np.einsum("hkv,hv->hk", left, dmiss)
            out["dq"][s, t], out["dk"][s, t], out["dv"][s, t] = dq, dk, dmiss
            out["dbeta"][s, t] = (du * miss).sum(1)
            out["dg"][s, t] = (dleft * left).sum((1, 2))
            lam = dleft * decay[s, t][:, None, None]
            mags = abs(lam) + abs(q[s, t][:, :, None] * d[:, None])
            du_mag = np.einsum("hkv,hk->hv", abs(at) + mags, abs(k[s, t]))
            miss_mag = abs(v[s, t]) + np.einsum("hkv,hk->hv", abs(left), abs(k[s, t]))
            dq_mag = np.einsum("hkv,hv->hk", abs(new), abs(d))
            dk_mag = np.einsum("hkv,hv->hk", abs(at), abs(u)) + np.einsum("hkv,hv->hk", abs(left), abs(beta[s, t][:, None]) * du_mag)
            largest("dq", s, dq_mag), largest("dk", s, dk_mag), largest("dv", s, abs(beta[s, t][:, None]) * du_mag)
            largest("dbeta", s, (du_mag * miss_mag).sum(1))
            row_sums = row_sums + (abs(q[s, t]) * dq_mag).sum(1) + (abs(v[s, t] * beta[s, t][:, None]) * du_mag).sum(1)
            largest("dg", s, row_sums + ends)
            largest("dh0", s, mags)
        out["dh0"][s] = lam
        first_cut = decay[s, 0] == 0
        out["dg"][s, 0][first_cut] = 0.0
        for t in range(1, length[s]):
            if not keep[s, t - 1]:
                out["dg"][s, t] = 0.0
    if back:
        for n in ("dq", "dk"):
            out[n] = out[n].reshape(S, T, Hk, share, Dk).sum(3)
            mag[n] = mag[n].reshape(S, Hk, share).sum(2)
        mag["dh0"] = np.maximum(mag["dh0"], 0.0 if dh_last is None else abs(dh_last).max((2, 3)))
    out.update({n + "_mag": m for n, m in mag.items()})
    return out


def delta_bound(n, want, Dk, Dv):
    """What output n of a 32-bit kernel may be off by, apart from its last rounding."""
    steps = (Dk + 3 * PIECE) * (1 if n in ("o", "h_last") else 2) + (0 if n in ("o", "h_last") else Dv)
    m = want[n + "_mag"]
    shape = {"o": (0, None, 1, None), "h_last": (0, 1, None, None), "dh0": (0, 1, None, None)}.get(n, (0, None, 1, None))
    return 2.0 ** -24 * steps * (m[:, None, :, None] if shape[1] is None else m[:, :, None, None])


def embedding(table, token, scale):
    named = (token >= 0) & (token < len(table))
    return np.where(named[:, None], table[np.where(named, token, 0)] * scale, 0.0)


def embedding_backward(dout, token, V, scale):
    """The gradient, and the sum of its terms' magnitudes."""
    named = (token >= 0) & (token < V)
    sums, mag, count = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V)
    np.add.at(sums, token[named], dout[named])
    np.add.at(mag, token[named], abs(dout[named]))
    np.add.at(count, token[named], 1)
    # a term goes through at most 63 sums of places ahead, 64 of a slice, 64 of slices, and as many as there are slices of slices
    depth = np.minimum(count, 3 * 64 + 63 + count / 4096)
    return sums * scale, mag * abs(scale) * (depth[:, None] + 1) * 2.0 ** -24


def clip(grads, max_norm):
    norm = np.sqrt(sum(float((np.asarray(x, np.float64) ** 2).sum()) for x in grads))
    factor = min(1.0, max_norm / norm) if np.isfinite(norm) and norm > 0 else 1.0
    return norm, [np.asarray(x, np.float64) * factor for x in grads]
