"""The distillation's loss and gradient from their definition in 80 bits, for students so near their teacher that the definition
cancels in 64, with bounds on what arithmetic may be off that holds sums over the vocabulary in 32 bits and does not cancel.
CPU only; test infrastructure.

With u = ln p - ln q for a named token, the loss is the sum of q (e^u - 1 - u), of the rest's like term, and of what the masses lack
of one another: an error of u, as of a common factor of all p, enters it times q (e^u - 1), not times q."""
import numpy as np

U = 2.0 ** -24
X = np.longdouble


def log_sum_exp(y):
    return y.max() + np.log(np.exp(y - y.max()).sum()) if len(y) and y.max() > -np.inf else X(-np.inf)


def distill(z, index, value, tau=1.0, top_lse=None, weight=None):
    """loss, lse, grad and their bounds (before the gradient's rounding); every row names distinct tokens within [0, V)."""
    N, V = z.shape
    out = {n: np.zeros(N) for n in ("loss", "lse", "loss_err", "lse_err")}
    out.update(grad=np.zeros((N, V)), grad_err=np.zeros((N, V)))
    for i in range(N):
        with np.errstate(divide="ignore"):
            named, y, v = index[i].astype(np.int64), z[i].astype(X) / X(tau), value[i].astype(X) / X(tau)
            lse = log_sum_exp(y)
            ln_p, ln_q = y - lse, v - (log_sum_exp(v) if top_lse is None else X(top_lse[i]))
            p, q = np.exp(ln_p), np.exp(ln_q)
            others = np.ones(V, bool)
            others[named] = False
            P, s, M = p[named].sum(), p[others].sum(), q.sum()
            r = max(X(0), 1 - M) if top_lse is not None and others.any() else X(0)
            loss = np.sum(np.where(q > 0, q * (ln_q - ln_p[named]), X(0))) + (r * (np.log(r) - np.log(s)) if r > 0 else X(0))
        factor = (M + r) - (r / s if r > 0 else 0)             # of the tokens that are not named
        grad = p * factor
        grad[named] = (M + r) * p[named] - q
        # a sum over the vocabulary: its terms one after the other in each of 512 threads, and their exponents' roundings
        span = y.max() - y
        span_o = np.where(others, y[others].max() - y, 0) if others.any() else np.zeros(V)
        e = float((V / 512 + 64 + np.sum(p * span) + 8) * U)
        apart = float(np.abs(p[named] - q).sum())              # sum of q |e^u - 1|
        if r > 0:
            first = apart + 4 * abs(float(P - M)) * float(1 + P / s)
            factor_err = 4 * abs(float(factor)) * (e + (2 * span + 2 * span_o + 32) * U) + float(r / s ** 2) * (float(P) * e + 8 * U * apart)
        else:
            first = apart + (0 if not others.any() else float(M))
            factor_err = float(M) * (e + (2 * span + 32) * U)
        g_err = p * factor_err
        g_err[named] = p[named] * e + 16 * U * (np.abs(p[named] - q) + abs(M + r - 1) * p[named])
        w = 1.0 if weight is None else float(weight[i])
        out["loss"][i], out["loss_err"][i] = loss, 2 * (e * first + e * e) + 16 * U * abs(float(loss))
        out["lse"][i], out["lse_err"][i] = lse, e + 8 * U * (abs(float(lse)) + abs(float(y.max())) + 1)
        out["grad"][i], out["grad_err"][i] = grad * w / tau, 2 * g_err * abs(w) / tau
    return out
