"""The label's own term of the gradients from hidden states of 16 bits, for more than 256 rows, whose g is rounded to
16 bits: the one large number of a row keeps what that rounding takes.

Bounds, with u = 2^-24 and half the half step of the type (2^-8 of bfloat16, 2^-11 of float16).  Where the upstream
gradients of the log-probability and of the log sum are the same number a, g is scale a at the label and 0 elsewhere.
The product of the rounded g and a weight is exact in float32; the rest, which is exact, is multiplied and added with a
rounding each, beside that of scale a and those of float16's power of two: 8 u.  For the weight's gradient the rest is
rounded to the type, half a step of what is half a step of g at most, and a class sums its rows in float32.  float16's
rest may lie among its smallest numbers, 2^-24 apart, where the largest |g| of all rows is 2^14 at least.
"""
import numpy as np
import pytest

import head_reference as ref
from gpu_util import announce
from test_gpu_head import make, numbers, run

pytestmark = pytest.mark.gpu

SIZES = [(257, 513, 96), (300, 513, 96), (300, 14, 2500), (1500, 20, 515), (1024, 2049, 1024), (2600, 700, 136),
         (4097, 130, 300), (700, 40, 1303), (3000, 1, 17)]


def bounds(g, hidden, weight, labels, dtype):
    """(dh, its bound, dw, its bound) of slopes g (N,) at the labels."""
    part = labels >= 0
    y = np.where(part, labels, 0)
    g = np.where(part, g, 0.0)
    dh = g[:, None] * weight[y]
    one = np.zeros((len(labels), weight.shape[0]))
    one[np.arange(len(labels)), y] = g
    dw, size = one.T @ hidden, np.abs(one).T @ np.abs(hidden)
    tol_w = (ref.HALF[dtype] ** 2 + 8 * ref.U + ref.walk(len(labels))) * size
    if dtype == "f16":
        tol_w += 2.0 ** -25 * 2.0 ** -14 * np.abs(g).max() * ((one != 0).T @ np.abs(hidden))
    return dh, 8 * ref.U * np.abs(dh), dw, tol_w


def label_alone(hidden, weight, labels, a, scale, dtype, what):
    import torch
    announce(what)
    n, v = hidden.shape[0], weight.shape[0]
    lost = (labels < 0) | (labels >= v)
    a = torch.where(lost, torch.zeros_like(a), a)
    _, (dh, dw) = run(hidden, weight, labels, [a, a], scale, True)
    y = torch.where(lost, torch.full_like(labels, -1), labels).cpu().numpy()
    g = float(np.float32(scale)) * numbers(a)
    want_h, tol_h, want_w, tol_w = bounds(g, numbers(hidden), numbers(weight), y, dtype)
    ref.check(numbers(dh), want_h, tol_h, "hidden's gradient", dtype)
    ref.check(numbers(dw), want_w, tol_w, "weight's gradient", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d", SIZES)
def test_label_alone(dtype, n, v, d):
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=3)
    label_alone(hidden, weight, labels, ups[0], 0.7, dtype, "label alone %s %dx%dx%d" % (dtype, n, v, d))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [((3, 5), (1, 1)), ((0, 8), (0, 0))])
def test_strides(dtype, pad, shift):
    hidden, weight, labels, ups = make(400, 300, 61, dtype, seed=3, pad=pad, shift=shift)
    label_alone(hidden, weight, labels, ups[0], 1.0, dtype, "label alone strides %s" % ((dtype, pad, shift),))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_class_has_all_labels(dtype):
    """More rows of one class than a workgroup lists at once, and none of most others."""
    import torch
    for n in (2111, 5000):
        hidden, weight, labels, ups = make(n, 600, 72, dtype, seed=4, missing=0.0)
        labels = torch.where(torch.arange(n, device="cuda") % 37 == 0, labels, torch.full_like(labels, 255))
        label_alone(hidden, weight, labels, ups[0], 1.0, dtype, "label alone, one class %s %d" % (dtype, n))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_pieces(dtype):
    """16384 rows: several pieces of the vocabulary, whose labels' terms are computed apart."""
    hidden, weight, labels, ups = make(16300, 9000, 64, dtype, missing=0.9)
    label_alone(hidden, weight, labels, ups[0], 1.0, dtype, "label alone, pieces " + dtype)


def test_wide_range_of_upstream_gradients():
    """float16 holds a row's g as a multiple of a power of two of its own, and all rows' of a common one."""
    import torch
    hidden, weight, labels, ups = make(600, 300, 64, "f16", seed=5)
    sizes = torch.logspace(-3, 3, 600, device="cuda")
    label_alone(hidden, weight, labels, ups[0] * sizes, 1.0, "f16", "label alone, range")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d", [(300, 513, 96), (1500, 20, 515), (2600, 700, 136)])
def test_beside_the_other_classes(dtype, n, v, d):
    """The bounds of head_reference, with the label's element of g at half a step of the rest instead of g's."""
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=6)
    announce("label beside others %s %dx%dx%d" % (dtype, n, v, d))
    _, (dh, dw) = run(hidden, weight, labels, ups, 1.0, False)
    h, w, y = numbers(hidden), numbers(weight), labels.cpu().numpy()
    want = ref.exact(h, w, y, 1.0, dtype, (numbers(ups[0]), None), False)
    has = (y >= 0) & (y < v)
    y0 = np.where(has, y, 0)
    x = (h @ w.T)[np.arange(n), y0]
    top = want["logp"]
    g = np.where(has, numbers(ups[0]) * (1 - np.exp(top)), 0.0)
    # what the general bound grants the label's element for its rounding, and what is left of it
    half = ref.HALF[dtype]
    spare = (half - half ** 2) * np.abs(g)
    one = np.zeros((n, v))
    one[np.arange(n), y0] = spare
    assert x.shape == (n,)
    ref.check(numbers(dh), want["dh"], want["tol_dh"] - one @ np.abs(w), "hidden's gradient", dtype)
    ref.check(numbers(dw), want["dw"], want["tol_dw"] - one.T @ np.abs(np.where(has[:, None], h, 0.0)), "weight's gradient", dtype)


def test_infinite_weights_keep_their_meaning():
    """A label whose weights hold -inf: its row's gradient is what the product makes of it, not NaN for the rest's sake."""
    import torch
    hidden, weight, labels, ups = make(300, 200, 40, "bf16", missing=0.0)
    hidden = hidden.abs() + 0.5
    weight[7, 3] = -float("inf")
    labels = torch.where(torch.arange(300, device="cuda") % 5 == 0, torch.full_like(labels, 7), labels % 7)
    announce("label of infinite weight")
    _, (dh, dw) = run(hidden, weight, labels, [ups[0].abs() + 1.01], 1.0, False)
    mine = labels == 7
    keep = torch.arange(40, device="cuda") != 3
    assert (dh[mine][:, 3] == -float("inf")).all()
    assert dh[mine][:, keep].isfinite().all() and dw[:7].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,d", [(300, 30, 300), (257, 128, 100), (1000, 17, 515), (4100, 9, 72), (600, 100, 1303)])
def test_few_classes(dtype, n, v, d, monkeypatch):
    """Of up to 128 classes each may be much of a row: g is the sum of two numbers for any number of rows."""
    monkeypatch.setitem(ref.HALF, dtype, ref.HALF[dtype] ** 2)
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=7)
    announce("few classes %s %dx%dx%d" % (dtype, n, v, d))
    _, (dh, dw) = run(hidden, weight, labels, ups, 1.0, False)
    want = ref.exact(numbers(hidden), numbers(weight), labels.cpu().numpy(), 1.0, dtype, (numbers(ups[0]), None), False)
    ref.check(numbers(dh), want["dh"], want["tol_dh"], "hidden's gradient", dtype)
    ref.check(numbers(dw), want["dw"], want["tol_dw"], "weight's gradient", dtype)
