"""The operators around the memory in 64 bits, step by step from their definitions, with bounds on what 32-bit arithmetic may be
off.  CPU only; test infrastructure."""
import numpy as np
import torch

U = 2.0 ** -24                          # unit roundoff of fp32
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -133), torch.float16: (2.0 ** -11, 2.0 ** -24)}
ONE = 1 << 40


def rounding(x, dtype):
    """What one rounding of x to `dtype` may change: half a unit in the last place, or half the smallest number."""
    rel, least = ROUND[dtype]
    return np.abs(x) * rel + least / 2


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


# -------------------------------------------------------------------------------------------------------------- scan

def gates(g, x, gate):
    """a, b, their derivatives' factor, and the relative error that a and b may have in fp32, in units of U."""
    if gate == "given":
        return g, x, np.zeros_like(g)
    with np.errstate(over="ignore"):
        a, rest = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    # the exponent of e^-|g| carries |g| units, its power, the sum, the reciprocal and two products some more
    return a, rest * x, np.abs(g) + 8


def scan(g, x, gate, discount=None, length=None, h0=None, dh=None, dh_last=None):
    """Everything of apex_gated_scan and its gradient, as a dict of float64 arrays, and the same names + "_err": bounds of the
    error before the outputs are rounded to their type.  Steps past a length and what an episode's end cuts are not looked at."""
    S, T, D = x.shape
    length = np.full(S, T) if length is None else np.clip(length, 0, T)
    ends = np.zeros((S, T), bool) if discount is None else np.asarray(discount) == 0
    out = {n: np.zeros((S, T, D)) for n in ("h", "h_err", "dg", "dg_err", "dx", "dx_err")}
    out.update({n: np.zeros((S, D)) for n in ("h_last", "h_last_err", "dh0", "dh0_err")})
    out["carry"] = np.full((S, -(-T // 64), D), np.nan)
    for s in range(S):
        n = int(length[s])
        a, b, k = gates(g[s, :n], x[s, :n], gate)
        state = np.zeros(D) if h0 is None else h0[s].copy()
        err, size = np.abs(state) * U, np.abs(state)        # size: the recurrence of absolute values
        prev, prev_err, prev_size = np.zeros((n, D)), np.zeros((n, D)), np.zeros((n, D))
        for t in range(n):
            if t % 64 == 0:
                out["carry"][s, t // 64] = state
            prev[t], prev_err[t], prev_size[t] = state, err, size
            now = a[t] * state + b[t]
            size = np.abs(a[t]) * size + np.abs(b[t])
            err = np.abs(a[t]) * err + (k[t] + 4) * U * size
            out["h"][s, t], out["h_err"][s, t] = now, 4 * err
            state = now
            if ends[s, t]:
                state, err, size = np.zeros(D), np.zeros(D), np.zeros(D)
        out["h_last"][s], out["h_last_err"][s] = state, 4 * err
        if dh is None:
            continue
        back = np.zeros(D) if dh_last is None else dh_last[s].copy()
        berr, bsize = np.abs(back) * U, np.abs(back)
        for t in reversed(range(n)):
            if ends[s, t]:
                back, berr, bsize = np.zeros(D), np.zeros(D), np.zeros(D)
            lam, lsize = dh[s, t] + back, np.abs(dh[s, t]) + bsize
            lerr = berr + 2 * U * lsize
            if gate == "given":
                dg, dx = lam * prev[t], lam
                dg_err = lerr * prev_size[t] + lsize * prev_err[t] + 4 * U * lsize * prev_size[t]
                dx_err = lerr
            else:
                rest = 1 / (1 + np.exp(g[s, t]))
                dg, dx = lam * (prev[t] - x[s, t]) * a[t] * rest, lam * rest
                both = prev_size[t] + np.abs(x[s, t])
                dg_err = (lerr * both + lsize * prev_err[t] + (2 * k[t] + 8) * U * lsize * both) * a[t] * rest
                dx_err = (lerr + (k[t] + 4) * U * lsize) * rest
            out["dg"][s, t], out["dg_err"][s, t] = dg, 4 * dg_err
            out["dx"][s, t], out["dx_err"][s, t] = dx, 4 * dx_err
            back, bsize = a[t] * lam, np.abs(a[t]) * lsize
            berr = np.abs(a[t]) * lerr + (k[t] + 4) * U * bsize
        out["dh0"][s], out["dh0_err"][s] = back, 4 * berr
    return out


# ----------------------------------------------------------------------------------------------------------- distill

def distill(z, index, value, tau=1.0, top_lse=None, weight=None):
    """loss, lse, grad and their bounds (before the gradient's rounding) of float64 arrays."""
    N, V = z.shape
    out = dict(loss=np.zeros(N), lse=np.zeros(N), grad=np.zeros((N, V)), loss_err=np.zeros(N), lse_err=np.zeros(N),
               grad_err=np.zeros((N, V)))
    for i in range(N):
        seen, named, v = set(), [], []
        for j, x in zip(index[i], value[i]):
            if 0 <= j < V and int(j) not in seen:
                seen.add(int(j))
                named.append(int(j))
                v.append(x / tau)
        named, v = np.array(named, np.int64), np.array(v, np.float64)
        y = z[i] / tau
        top = y.max()
        with np.errstate(all="ignore"):
            lse = top + np.log(np.exp(y - top).sum())
            log_p = y - lse
            p = np.exp(log_p)
            if top_lse is not None:
                log_q = v - top_lse[i]
            else:
                log_q = v - (v.max() + np.log(np.exp(v - v.max()).sum())) if len(v) and v.max() > -np.inf else np.full(len(v), -np.inf)
            q = np.exp(log_q)
            # a power carries its exponent's rounding; a sum that of its terms, one after the other in each of 512 threads
            span = np.where(np.isfinite(y), np.abs(y - top), 0.0)
            eS = (V / 512 + 64 + np.sum(p * span)) * U
            terms = np.where(q > 0, q * (log_q - log_p[named]), 0.0)
            eq = (np.where(np.isfinite(v), np.abs(v - (v.max() if len(v) else 0)), 0) + np.abs(np.where(q > 0, log_q, 0)) + len(v) + 16) * U
            loss = terms.sum()
            loss_err = np.sum(np.where(q > 0, q * (eq * (1 + np.abs(log_q - log_p[named])) + eS + (np.abs(log_p[named]) + 8) * U), 0))
            M = q.sum()
            g = M * p
            g[named] -= q
            g_err = M * p * (eS + (span + 16 + len(v)) * U)
            g_err[named] += q * (eq + 8 * U)
            if top_lse is not None and len(named) < V:
                r = max(0.0, 1.0 - M)
                others = np.ones(V, bool)
                others[named] = False
                so = p[others].sum()
                r_err = np.sum(q * eq) + 4 * U
                if r > 0:
                    yo = np.where(others, y, -np.inf)
                    lse_o = yo.max() + np.log(np.exp(yo - yo.max()).sum()) if yo.max() > -np.inf else -np.inf
                    loss += r * (np.log(r) - (lse_o - lse))
                    loss_err += r_err * (1 + abs(np.log(r) - (lse_o - lse))) + r * (2 * eS + (abs(lse_o - lse) + 16) * U)
                    po = np.exp(yo - lse_o) if lse_o > -np.inf else np.zeros(V)
                    g += r * p - r * po
                    g_err += (r_err + r * (2 * eS + (2 * span + 32) * U)) * (p + po)
                else:
                    po = np.exp(np.where(others, y, -np.inf) - top) / np.exp(np.where(others, y, -np.inf) - top).sum() if so > 0 else np.zeros(V)
                    g_err += r_err * (p + po)
            w = 1.0 if weight is None else weight[i]
            out["loss"][i], out["loss_err"][i] = loss, 2 * loss_err + 1e-30
            out["lse"][i], out["lse_err"][i] = lse, eS + 8 * U * (abs(lse) + abs(top) + 1)
            out["grad"][i] = g * w / tau if w != 0 else 0.0
            out["grad_err"][i] = 2 * g_err * abs(w) / tau
    return out


# ------------------------------------------------------------------------------------------------------------ verify

def masses(x):
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        return np.floor(np.where(x > 0, np.minimum(x, 1.0), 0.0) * ONE).astype(np.int64)


def verify(target, draft, token, rnd, length=None):
    """accepted [B] and token [B,G+1]; rnd as uint64."""
    B, G = target.shape[0], target.shape[1] - 1
    V = target.shape[2]
    accepted, out = np.zeros(B, np.int32), np.full((B, G + 1), -1, np.int32)
    for b in range(B):
        n, top = 0, G if length is None else min(max(int(length[b]), 0), G)
        while n < top:
            t = int(token[b, n])
            if not 0 <= t < V:
                break
            p, q = int(masses(target[b, n, t])), int(masses(draft[b, n, t]))
            if not (int(rnd[b, n]) * q) >> 64 < p:
                break
            out[b, n] = t
            n += 1
        m = p = masses(target[b, n])
        if n < top:
            m = np.maximum(p - masses(draft[b, n]), 0)
            m = m if m.any() else p
        up_to = np.cumsum(m)
        if up_to[-1]:
            out[b, n] = np.searchsorted(up_to, (int(rnd[b, G]) * int(up_to[-1])) >> 64, side="right")
        accepted[b] = n
    return accepted, out
