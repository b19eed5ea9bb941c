"""Biases by buckets of distance in numpy, from the definition: float32 distances with every
operation rounded, buckets by comparison, values and sums in float64."""
import itertools

import numpy as np

U = 2.0 ** -24
HALF_ULP = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}


def grid_distances(query, key, offset, metric, sampling):
    place = [np.array(list(itertools.product(*[range(n) for n in shape])), np.int64).reshape(-1, len(shape))
             for shape in (query, key)]
    delta = (place[1][None] - (place[0] + np.asarray(offset))[:, None]).astype(np.float32)
    if metric == "offset":
        return delta[..., 0]
    if sampling is not None:
        delta = delta * np.asarray(sampling, np.float32)
    terms = delta * delta if metric == "euclidean" else np.abs(delta)
    total = terms[..., 0]
    for a in range(1, len(query)):
        total = np.maximum(total, terms[..., a]) if metric == "chessboard" else (total + terms[..., a]).astype(np.float32)
    return np.sqrt(total) if metric == "euclidean" else total


def buckets(distance, edges):
    d = np.asarray(distance).astype(np.float32)
    out = np.zeros(d.shape, np.int64)
    with np.errstate(invalid="ignore"):
        for e in np.asarray(edges, np.float32):
            out += e <= d
    return out


def forward(table, bucket, add=None):
    """bucket (B, P) -> (B, H, P) float64."""
    value = np.asarray(table, np.float64)[bucket]                # (B, P, H)
    value = value.transpose(0, 2, 1)
    return value if add is None else value + add


def gradient(up, bucket, count):
    """up (B, H, P), bucket (B or 1, P): sums per bucket and head, and sums of magnitudes."""
    bucket = np.broadcast_to(bucket, (up.shape[0], up.shape[2]))
    total = np.zeros((count, up.shape[1]))
    size = np.zeros((count, up.shape[1]))
    number = np.bincount(bucket.reshape(-1), minlength=count)
    for b in range(up.shape[0]):
        for h in range(up.shape[1]):
            with np.errstate(invalid="ignore"):
                total[:, h] += np.bincount(bucket[b], up[b, h], count)
                size[:, h] += np.bincount(bucket[b], np.abs(up[b, h]), count)
    return total, size, number


def check(got, want, tol, dtype, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    rel, sub = HALF_ULP[dtype]
    tol = np.broadcast_to(tol, want.shape) + rel * (np.abs(np.where(np.isfinite(want), want, 0)) + tol) + sub
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r, want %r" % (
        what, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), got[tuple(np.argwhere(bad)[0])],
        want[tuple(np.argwhere(bad)[0])])
