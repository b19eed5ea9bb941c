"""Label log-probabilities, their companions and gradients in float64 numpy, straight from
the definitions, with the rounding error that float32 arithmetic may leave.

Bounds.  With u = 2^-24, a logarithm of a sum of C positive terms computed in float32 is off by
at most u (8 + 8 sqrt C) in absolute terms: each exponential carries a few u and the error of its
argument, whose weighted mean over the classes is a few u; the additions' roundings, independent
and in no order that matters here, add up like a random walk, for which 8 sqrt C is far out.  A
log-probability l adds u per operation relative to |l| and to |x - max|.  Everything made from
probabilities inherits that bound relatively.
"""
import numpy as np

U = 2.0 ** -24


def exact(logits, labels, field=None, top_k=0, ups=None):
    """logits (N, C) float64 (the values that the kernel reads), labels (N,) ints, field (N, C).
    ups: (a, h, f), each (N,) or None.  Returns a dict with values and "tol_..." bounds."""
    x = np.asarray(logits, np.float64)
    n, classes = x.shape
    alive = np.isfinite(x).any(1)
    with np.errstate(all="ignore"):
        m = np.where(alive, np.nanmax(np.where(np.isneginf(x), -np.inf, x), 1), 0.0)
        e = np.exp(x - m[:, None])
        s = e.sum(1)
        l = np.where(alive[:, None], x - m[:, None] - np.log(s)[:, None], -np.inf)
        p = np.exp(l)
        lz = np.where(p > 0, l, 0.0)
        has = (labels >= 0) & (labels < classes)
        y = np.where(has, labels, 0)
        out = {"logp": np.where(has, l[np.arange(n), y], 0.0), "entropy": -(p * lz).sum(1)}
    base = U * (8 + 8 * np.sqrt(classes))
    spread = np.abs(lz).max(1)
    finite_logp = np.where(np.isfinite(out["logp"]), out["logp"], 0.0)
    out["tol_logp"] = base + 4 * U * np.abs(finite_logp)
    # sum p |l - l~| + |l| |p - p~|, each off by base + 4 u |l| (absolutely, relatively)
    weight = (p * (1 + np.abs(lz)) * (base + 4 * U * np.abs(lz))).sum(1)
    out["tol_entropy"] = 2 * weight + base + 4 * U * out["entropy"]
    if field is not None:
        phi = np.where(p > 0, field, 0.0).astype(np.float64)
        out["mean"] = (p * phi).sum(1)
        out["tol_mean"] = 2 * (p * np.abs(phi) * (base + 4 * U * np.abs(lz))).sum(1) + base * np.abs(out["mean"])
    if top_k:
        order = np.argsort(-x, axis=1, kind="stable")[:, :top_k]
        out["index"] = order
        out["top"] = np.take_along_axis(l, order, 1)
        out["tol_top"] = base + 4 * U * np.abs(np.where(np.isfinite(out["top"]), out["top"], 0.0))
    if ups is not None:
        a, h, f = ups
        grad = np.zeros_like(x)
        tol = np.zeros_like(x)
        rel = base + 4 * U * np.abs(lz) + 4 * U
        if a is not None:
            au = np.where(has & alive, a, 0.0)
            one = np.zeros_like(x)
            one[np.arange(n), y] = 1
            grad += au[:, None] * (one - p)
            tol += np.abs(au)[:, None] * (p * rel + 4 * U * one)
        if h is not None:
            hz = out["entropy"]
            grad -= h[:, None] * p * (lz + hz[:, None])
            tol += np.abs(h)[:, None] * p * ((np.abs(lz) + hz[:, None]) * rel + base + 4 * U * np.abs(lz)
                                             + out["tol_entropy"][:, None])
        if f is not None:
            grad += f[:, None] * p * (phi - out["mean"][:, None])
            tol += np.abs(f)[:, None] * p * ((np.abs(phi) + np.abs(out["mean"])[:, None]) * rel
                                             + out["tol_mean"][:, None])
        out["grad"], out["tol_grad"] = np.where(alive[:, None], grad, 0.0), tol
    out["spread"] = spread
    return out


# One rounding to the output's type: half a unit in the last place, and half the spacing of its subnormals.
ROUND = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}


def check(got, want, tol, what, dtype=None):
    got = np.asarray(got, np.float64)
    want = np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    finite = np.isfinite(want)
    assert np.array_equal(got[~finite], want[~finite]), "%s: infinities differ" % what
    # exponentials below 2^-126 flush to zero
    tol = np.broadcast_to(tol, want.shape) + 2.0 ** -120
    if dtype:
        rel, sub = ROUND[dtype]
        tol = tol + rel * (np.abs(want) + tol) + sub
    err = np.abs(np.where(finite, got - np.where(finite, want, 0.0), 0.0))
    bad = ~(err <= tol) & finite
    assert not bad.any(), "%s: %d of %d off, worst %.3g of a bound of %.3g at %s" % (
        what, bad.sum(), bad.size, err[bad].max(), tol[bad][err[bad].argmax()], tuple(np.argwhere(bad)[0]))
