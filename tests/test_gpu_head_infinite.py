"""Float32 log-probabilities from hidden states with infinities and the largest numbers among the operands, for numbers of
rows that take every way to the matrix cores: an infinite bias column takes classes out, a number is never lost to NaN."""
import numpy as np
import pytest

import head_reference as ref
from gpu_util import announce
from test_gpu_head import make, numbers, run

pytestmark = pytest.mark.gpu

# single waves, narrow and plain tiles of floats, planes with g by single waves, planes by tiles of both sizes
SIZES = [(12, 300, 40), (100, 300, 40), (60, 9000, 1100), (120, 9000, 1100), (300, 300, 40), (1100, 1000, 600),
         (700, 17000, 200)]


def with_bias(n, v, d, lowest):
    """Hidden states with a last column of ones, beside a bias that is `lowest` for every third class and 0 for others."""
    import torch
    hidden, weight, labels, ups = make(n, v, d, "f32", seed=8, missing=0.1)
    hidden[:, -1] = 1.0
    weight[:, -1] = 0.0
    banned = torch.arange(v, device="cuda") % 3 == 1
    weight[banned, -1] = lowest
    valid = (labels >= 0) & (labels < v)
    labels = torch.where(valid, labels // 3 * 3, labels)
    return hidden, weight, labels, ups, banned


@pytest.mark.parametrize("n,v,d", SIZES)
@pytest.mark.parametrize("lowest", [float("-inf"), float(np.finfo(np.float32).min), -3.395e38])
def test_banned_classes(n, v, d, lowest):
    import torch
    announce("banned classes %dx%dx%d %g" % (n, v, d, lowest))
    hidden, weight, labels, ups, banned = with_bias(n, v, d, lowest)
    got, (dh, dw) = run(hidden, weight, labels, ups, 1.0, True)
    left = (~banned).cpu().numpy()
    y = labels.cpu().numpy()
    valid = (y >= 0) & (y < v)
    place = np.cumsum(left) - 1
    y = np.where(valid, place[np.where(valid, y, 0)], -1)
    want = ref.exact(numbers(hidden), numbers(weight)[left], y, 1.0, "f32", (numbers(ups[0]), numbers(ups[1])), True)
    ref.check(numbers(got.log_probs), want["logp"], want["tol_logp"], "log_probs")
    ref.check(numbers(got.log_sums), want["log_sum"], want["tol_log_sum"], "log_sums")
    # 0 x -inf is no number, in the bias column alone
    cut = d - 1 if lowest == float("-inf") else d
    ref.check(numbers(dh)[:, :cut], want["dh"][:, :cut], want["tol_dh"][:, :cut], "hidden's gradient")
    ref.check(numbers(dw)[left], want["dw"], want["tol_dw"], "weight's gradient")
    assert not dw[banned].any()


@pytest.mark.parametrize("n,v,d", SIZES)
def test_banned_labels(n, v, d):
    import torch
    announce("banned labels %dx%dx%d" % (n, v, d))
    from paper_2608_24738_amd import training
    hidden, weight, labels, _, banned = with_bias(n, v, d, float("-inf"))
    labels = torch.where(torch.arange(n, device="cuda") % 2 == 0, torch.full_like(labels, 1), labels)
    got = training.head_log_probs(hidden, weight, labels, log_sums=True)
    assert (got.log_probs[::2] == -float("inf")).all() and got.log_probs[1::2].isfinite().all()
    assert got.log_sums.isfinite().all()
    weight[:, -1] = -float("inf")
    got = training.head_log_probs(hidden, weight, torch.zeros_like(labels), log_sums=True)
    assert (got.log_probs == -float("inf")).all() and (got.log_sums == -float("inf")).all()


@pytest.mark.parametrize("n,v,d", SIZES)
def test_infinite_and_nan_rows(n, v, d):
    """A row with +inf among its logits, or NaN, is NaN, and no other row changes."""
    import torch
    announce("infinite rows %dx%dx%d" % (n, v, d))
    from paper_2608_24738_amd import training
    hidden, weight, labels, _, _ = with_bias(n, v, d, 0.0)
    labels = labels.clamp(0, v - 1)
    base = training.head_log_probs(hidden, weight, labels, log_sums=True)
    dirty = hidden.clone()
    dirty[2, 5], dirty[7, 0], dirty[9, 3] = float("inf"), float("nan"), -float("inf")
    got = training.head_log_probs(dirty, weight, labels, log_sums=True)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[[2, 7, 9]] = True
    for a, b in zip(got, base):
        assert a[bad].isnan().all() and torch.equal(a[~bad], b[~bad])


@pytest.mark.parametrize("n,v,d", SIZES)
@pytest.mark.parametrize("most", [float(np.finfo(np.float32).max), -3.395e38])
def test_largest_numbers(n, v, d, most):
    """Hidden states near the largest float32 beside small weights: ordinary logits."""
    announce("largest numbers %dx%dx%d %g" % (n, v, d, most))
    hidden, weight, labels, ups = make(n, v, d, "f32", seed=9)
    hidden[::2, 1] = most
    weight *= 1e6
    weight[:, 1] *= 1e-38
    got, _ = run(hidden, weight, labels, ups, 1e-6, True)
    want = ref.exact(numbers(hidden), numbers(weight), labels.cpu().numpy(), 1e-6, "f32", None, True)
    ref.check(numbers(got.log_probs), want["logp"], want["tol_logp"], "log_probs")
    ref.check(numbers(got.log_sums), want["log_sum"], want["tol_log_sum"], "log_sums")
