"""Log-probabilities from hidden states, and their gradients, in float64 numpy straight from the definitions, with
the rounding error that the kernels may leave.

Bounds, with u = 2^-24.  A float32 sum of d products is off by at most u (8 + 4 sqrt d) times the sum of their sizes:
the additions' roundings are independent and add up like a random walk, for which that is far out.  Let x be the
largest such error of a row's logits and X its largest logit: probabilities are off by 2 x relatively, by the rounding
of the factor log2(e), 2 u X, and by that of a sum of V terms, u (8 + 8 sqrt V).  A slope g is rounded to the operands'
type (half a step; of float16 also half the spacing of its smallest numbers, after the powers of two), and the products
with it are again float32 sums.  For 5 to 256 rows of 16 bits it is the sum of two such numbers: the second is the
rounding of what the first leaves, which is half a step at most, so half a step of it is half a step squared (2^-16 of
bfloat16, 2^-22 of float16).  For fewer it is kept in float32.

Exponentials below 2^-126 flush to zero, and so do operands of a product below that: p and then g lose up to 2^-126
each, which times |w| or |h| and summed is far above a float32's smallest numbers where those are in the hundreds.
"""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
STORE = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


def walk(n, factor=4):
    return U * (8 + factor * np.sqrt(n))


def exact(hidden, weight, labels, scale, dtype, ups=None, all_rows=False):
    """hidden (N, D), weight (V, D) float64, labels (N,) ints or None, ups (a, z), each (N,) or None."""
    h, w = np.asarray(hidden, np.float64), np.asarray(weight, np.float64)
    scale = float(np.float32(scale))
    n, v = h.shape[0], w.shape[0]
    y = np.full(n, -1) if labels is None else np.asarray(labels, np.int64)
    has = (y >= 0) & (y < v)
    part = has | all_rows
    y0 = np.where(has, y, 0)
    hz = np.where(part[:, None], h, 0.0)
    x = scale * (hz @ w.T)
    ex = (scale * walk(h.shape[1]) * (np.abs(hz) @ np.abs(w).T)).max(1)
    top = x.max(1)
    total = top + np.log(np.exp(x - top[:, None]).sum(1))
    rel = 2 * ex + 2 * U * np.abs(x).max(1) + walk(v, 8)
    out = {"log_sum": total, "tol_log_sum": rel + 4 * U * np.abs(total)}
    logp = np.where(has, x[np.arange(n), y0] - total, 0.0)
    out["logp"], out["tol_logp"] = logp, np.where(has, rel + 4 * U * np.abs(logp), 0.0)
    if ups is None:
        return out
    a = np.where(has, 0.0 if ups[0] is None else ups[0], 0.0)
    z = np.zeros(n) if ups[1] is None else np.asarray(ups[1], np.float64)
    p = np.exp(x - total[:, None])
    one = np.zeros_like(x)
    one[np.arange(n), y0] = has
    g = scale * (a[:, None] * one - (a - z)[:, None] * p)
    g[~part] = 0.0
    tol = scale * (np.abs(a - z)[:, None] * p * (rel[:, None] + 8 * U) + 4 * U * np.abs(a)[:, None] * one)
    tol += 2.0 ** -126 * (1 + scale * np.abs(a - z))[:, None]
    tol[~part] = 0.0
    few = n <= 4 or (dtype == "f32" and n <= 16)
    size = scale * (np.abs(a) + np.abs(a - z))
    if few:
        tol_w = tol_h = tol
    else:
        half = HALF[dtype] ** 2 if n <= 256 else HALF[dtype]
        tol_h = tol + half * (np.abs(g) + tol)
        tol_w = tol_h
        if dtype == "f16":
            # numbers below 2^-14 of the scaled slopes lie 2^-24 apart; sizes are brought to 2^14 at least
            tol_h = tol_h + 2.0 ** -25 * 2.0 ** -14 * size[:, None]
            tol_w = tol_w + 2.0 ** -25 * 2.0 ** -14 * size.max() * part[:, None]
    aw, ah = np.abs(w), np.abs(hz)
    out["dh"] = g @ w
    out["tol_dh"] = tol_h @ aw + walk(v) * (np.abs(g) @ aw)
    out["dw"] = g.T @ hz
    out["tol_dw"] = tol_w.T @ ah + walk(n) * (np.abs(g).T @ ah)
    return out


def check(got, want, tol, what, dtype="f32"):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    tol = tol + STORE[dtype] * (np.abs(want) + tol) + LEAST[dtype] + 2.0 ** -120
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first %s: %r for %r within %.3g" % (
        what, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), got[bad][0], want[bad][0], tol[bad][0])
