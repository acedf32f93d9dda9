"""The 80-bit form of the distillation against the 64-bit one and against its own terms that do not cancel (no GPU)."""
import numpy as np

import divergence_plain as near
import operators_plain as plain


def test_agrees_with_the_definition_in_64_bits():
    rng = np.random.default_rng(1)
    z, t = rng.standard_normal((5, 300)), rng.standard_normal((5, 300))
    index = np.stack([rng.permutation(300)[:7] for _ in range(5)])
    value, weight = np.take_along_axis(t, index, 1), rng.uniform(0.1, 1, 5)
    for lse in (None, np.log(np.exp(t / 1.5).sum(1))):
        a, b = near.distill(z, index, value, 1.5, lse, weight), plain.distill(z, index, value, 1.5, lse, weight)
        for n in ("loss", "lse", "grad"):
            assert np.abs(a[n] - b[n]).max() < 1e-12, n


def test_is_the_sum_of_terms_that_are_not_negative():
    """Where masses are whole: sum of q (e^u - 1 - u), rest included, for students from far to 1e-4 away."""
    rng = np.random.default_rng(2)
    for apart in (1.0, 1e-2, 1e-4):
        z = rng.standard_normal((3, 5000))
        t = z + rng.standard_normal(z.shape) * apart
        index = np.argsort(-t, axis=1)[:, :3]
        value = np.take_along_axis(t, index, 1)
        got = near.distill(z, index, value, 2.0, np.log(np.exp(t / 2).sum(1)))
        for i in range(3):
            ln_p, ln_q = (a[i] / 2 - np.log(np.exp(a[i] / 2).sum()) for a in (z, t))
            j = index[i]
            others = np.setdiff1d(np.arange(5000), j)
            u = np.append((ln_p - ln_q)[j], np.log(np.exp(ln_p[others]).sum()) - np.log(np.exp(ln_q[others]).sum()))
            q = np.append(np.exp(ln_q)[j], np.exp(ln_q[others]).sum())
            phi = np.where(np.abs(u) < 1e-3, u * u / 2 + u ** 3 / 6 + u ** 4 / 24, np.expm1(u) - u)
            assert abs((q * phi).sum() - got["loss"][i]) < 1e-8 * got["loss"][i] + 1e-18, (apart, i)
