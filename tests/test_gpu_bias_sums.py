"""The gradient of a bias's table where its sums are long, against sums in float64.

Bounds.  With u = 2^-24, a sum of positive terms is off by at most u of itself for every addition that a term goes
through.  The positions of 16 heads are spread over the waves of up to 512 workgroups, 4096 in all, but for a last
step of up to 512 positions to a wave; a wave's sum takes every position of it, float32 ones in three pieces; behind it
come 8 waves, 32 workgroups and 4 halvings: u (3 (positions / 4096 + 512) + 44) of the sum for any order of additions.
"""
import numpy as np
import pytest

import bias_reference as ref
from gpu_util import announce

pytestmark = pytest.mark.gpu

TYPES = {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}
U = 2.0 ** -24


def bound(positions):
    return U * (3 * (positions / 4096 + 512) + 44)


def field_gradient(d, edges, up, heads):
    import torch
    from paper_2608_24738_amd import training
    table = torch.zeros((edges.numel() + 1, heads), device=d.device, requires_grad=True)
    bias = training.distance_bias(d, table, edges, add=up)
    return torch.autograd.grad([bias], [table], [up])[0].double().cpu().numpy()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads", [1, 3, 16, 20])
@pytest.mark.parametrize("batch,shape", [(70001, ()), (1 << 20, ()), (70001, (3,)), (1 << 18, (3,)), (100003, (7,)),
                                         (3, (350003,))])
def test_equal_gradients(batch, shape, heads, dtype):
    """Equal gradients, which no binary number of few bits is, in three buckets, one of them of nearly all elements."""
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    gen = torch.Generator().manual_seed(batch)
    d = torch.where(torch.rand((batch,) + shape, generator=gen) < 0.9, 2.0, 30 * torch.rand((batch,) + shape, generator=gen))
    edges = torch.tensor([1.0, 15.0])
    announce("equal gradients %d x %s, %d heads, %s" % (batch, shape, heads, dtype))
    up = torch.full((batch, heads) + shape, 0.1, dtype=getattr(torch, TYPES[dtype]), device=dev)
    got = field_gradient(d.to(dev), edges.to(dev), up, heads)
    number = np.bincount(ref.buckets(d.numpy(), edges.numpy()).reshape(-1), minlength=3)
    want = np.repeat((number * float(up.reshape(-1)[0]))[:, None], heads, 1)
    ref.check(got, want, bound(d.numel()) * want, "f32", "equal gradients")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("positions", [1, 2, 3, 4, 5, 7, 8, 9])
@pytest.mark.parametrize("batch,heads,buckets", [(1, 1, 1), (2, 5, 9), (63, 16, 40), (64, 4, 256), (65, 33, 17),
                                                 (1001, 2, 130)])
def test_small_samples(batch, heads, buckets, positions, dtype):
    """Samples of fewer positions than one load, and about as many; fields of their own, and a grid that all share."""
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    gen = torch.Generator().manual_seed(batch + positions)
    kind = getattr(torch, TYPES[dtype])
    edges = training.distance_edges(buckets, 40)
    announce("small samples %d x %d, %d heads, %d buckets, %s" % (batch, positions, heads, buckets, dtype))
    d = torch.rand((batch, positions), generator=gen) * 40
    up = torch.randn((batch, heads, positions), generator=gen).to(kind)
    got = field_gradient(d.to(dev), edges.to(dev), up.to(dev), heads)
    total, size, _ = ref.gradient(up.double().numpy(), ref.buckets(d.numpy(), edges.numpy()), buckets)
    ref.check(got, total, 16 * U * size, "f32", "fields")
    table = torch.zeros((buckets, heads), device=dev, requires_grad=True)
    scores = up.reshape(batch, heads, 1, positions).to(dev)
    bias = training.relative_bias(table, edges.to(dev), 1, positions, query_offset=3, metric="taxicab", add=scores)
    got, = torch.autograd.grad([bias], [table], [scores])
    bucket = ref.buckets(ref.grid_distances((1,), (positions,), (3,), "taxicab", None), edges.numpy()).reshape(1, -1)
    total, size, _ = ref.gradient(up.double().numpy(), bucket, buckets)
    ref.check(got.double().cpu().numpy(), total, 16 * U * size, "f32", "a grid")
