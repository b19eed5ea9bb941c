"""The training operators where offsets pass 2^32 elements, at a few places against the definitions in float64."""
import numpy as np
import pytest

import bias_reference
import label_reference as ref
from gpu_util import announce

pytestmark = pytest.mark.gpu


def test_large_maps():
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    classes, n = 3, 1500000011
    announce("label_log_probs (1, %d, %d) bf16" % (classes, n))
    x = torch.empty((1, classes, n), dtype=torch.bfloat16, device=dev).uniform_(-4, 4)
    y = torch.empty((1, n), dtype=torch.uint8, device=dev).random_(0, classes + 1)
    up = torch.empty((1, n), device=dev).uniform_(-1, 1)
    x.requires_grad_(True)
    got = training.label_log_probs(x, y, top_k=1)
    grad, = torch.autograd.grad([got.log_probs], [x], [up])
    for at in (0, 12345, n // 2, 2 ** 30 + 3, n - 9, n - 1):
        want = ref.exact(x.detach()[:, :, at].double().cpu().numpy(), y[:, at].long().cpu().numpy(), top_k=1,
                         ups=[up[:, at].double().cpu().numpy(), None, None])
        ref.check(got.log_probs.detach()[:, at].cpu(), want["logp"], want["tol_logp"], "log_probs at %d" % at)
        assert int(got.top_indices[0, 0, at]) == int(want["index"][0, 0])
        ref.check(grad[:, :, at].double().cpu().numpy(), want["grad"], want["tol_grad"], "gradient at %d" % at, "bf16")


def test_large_rows():
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    n, classes = 70001, 65537
    announce("label_log_probs (%d, %d) bf16" % (n, classes))
    x = torch.empty((n, classes), dtype=torch.bfloat16, device=dev).uniform_(-4, 4)
    y = torch.empty(n, dtype=torch.int64, device=dev).random_(0, classes)
    up = torch.empty(n, device=dev).uniform_(-1, 1)
    x.requires_grad_(True)
    got = training.label_log_probs(x, y, entropy=True, top_k=2)
    grad, = torch.autograd.grad([got.log_probs, got.entropy], [x], [up, up])
    rows = [0, 1, 65535, 65536, n - 1]
    u = up[rows].double().cpu().numpy()
    want = ref.exact(x.detach()[rows].double().cpu().numpy(), y[rows].cpu().numpy(), top_k=2, ups=[u, u, None])
    ref.check(got.log_probs.detach()[rows].cpu(), want["logp"], want["tol_logp"], "log_probs")
    ref.check(got.entropy.detach()[rows].cpu(), want["entropy"], want["tol_entropy"], "entropy")
    assert np.array_equal(got.top_indices[rows].cpu().numpy(), want["index"])
    ref.check(grad[rows].double().cpu().numpy(), want["grad"], want["tol_grad"], "gradient", "bf16")


def test_many_short_rows():
    """More rows of a wave each than one dimension of a grid has threads for."""
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    n, classes = 2 ** 26 + 1001, 66
    announce("label_log_probs (%d, %d) bf16" % (n, classes))
    x = torch.empty((n, classes), dtype=torch.bfloat16, device=dev).uniform_(-4, 4)
    y = torch.empty(n, dtype=torch.uint8, device=dev).random_(0, classes)
    up = torch.empty(n, device=dev).uniform_(-1, 1)
    x.requires_grad_(True)
    got = training.label_log_probs(x, y)
    grad, = torch.autograd.grad([got.log_probs], [x], [up])
    rows = [0, 1, 2 ** 23, 2 ** 26 - 1, 2 ** 26, n - 1]
    want = ref.exact(x.detach()[rows].double().cpu().numpy(), y[rows].long().cpu().numpy(),
                     ups=[up[rows].double().cpu().numpy(), None, None])
    ref.check(got.log_probs.detach()[rows].cpu(), want["logp"], want["tol_logp"], "log_probs")
    ref.check(grad[rows].double().cpu().numpy(), want["grad"], want["tol_grad"], "gradient", "bf16")


def test_large_bias():
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    heads, length = 40, 11003
    announce("relative_bias %d x %d x %d bf16" % (heads, length, length))
    edges = training.distance_edges(32, length, signed=True)
    table = torch.randn((32, heads), device=dev).to(torch.bfloat16).requires_grad_(True)
    bias = training.relative_bias(table, edges.to(dev), length, length, metric="offset")
    up = torch.zeros((heads, length, length), dtype=torch.bfloat16, device=dev)
    want = np.zeros((32, heads))
    rng = np.random.default_rng(3)
    for h in (0, 17, 38, 39):
        for q, k in rng.integers(0, length, (40, 2)).tolist() + [[0, 0], [length - 1, length - 1], [length - 1, 0]]:
            bucket = int(bias_reference.buckets(np.float32(k - q), edges.numpy()))
            assert float(bias[h, q, k]) == float(table[bucket, h])
            value = float(rng.integers(1, 9))
            want[bucket, h] += value - float(up[h, q, k])
            up[h, q, k] = value
    grad, = torch.autograd.grad([bias], [table], [up])
    # sums of small whole numbers: exact before the rounding to bfloat16
    bias_reference.check(grad.double().cpu().numpy(), want, 0.0, "bf16", "gradient")
