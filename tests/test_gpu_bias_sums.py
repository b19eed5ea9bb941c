"""The gradient of a bias's table where its sums are long or not finite, against sums in float64.

Bounds.  With u = 2^-24, a sum of positive terms is off by at most u of itself for every addition that a term goes
through.  The positions of 16 heads are spread over the waves of up to 512 workgroups, 4096 in all (half as many for
20 heads, whose shares stay below the second term here), but for a last step of up to 512 positions to a wave; a wave's
sum takes every position of it, float32 ones in three pieces; behind it come 8 waves, 32 workgroups and 4 halvings:
u (3 (positions / 4096 + 512) + 44) of the sum for any order of additions.
"""
import time

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
@pytest.mark.parametrize("batch,positions,heads", [(32, 1 << 20, 1), (8, 1 << 20, 3), (5, 1 << 19, 16)])
def test_long_sums(batch, positions, heads, dtype):
    """Many equal gradients.  Their first 8 bits (16-bit ones have 11 at most) add up exactly while a wave has no more
    than 2^13 of them, 2^25 to 4096 waves.  What is left of float32 ones is below 2^-7 of them in two pieces: 512
    products of 32 positions, of 8 additions each, that round by half of 2^-23 of a sum which grows evenly, 2^-24 of its
    last value on average, are 4096 u 2^-7 = 32 u; 20 more for the waves and workgroups, each by half a unit."""
    import torch
    dev = "cuda:0"
    announce("long sums %d x %d, %d heads, %s" % (batch, positions, heads, dtype))
    d = torch.full((batch, positions), 7.0, device=dev)
    up = torch.full((batch, heads, positions), 0.1, dtype=getattr(torch, TYPES[dtype]), device=dev)
    got = field_gradient(d, torch.tensor([1.0, 15.0], device=dev), up, heads)
    want = np.zeros((3, heads))
    want[1] = float(up[0, 0, 0]) * batch * positions
    ref.check(got, want, 52 * U * want, "f32", "long sums")


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


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,buckets", [(1, 5), (3, 24), (6, 17), (16, 32), (20, 70), (5, 256)])
@pytest.mark.parametrize("positions", [1, 3, 7, 9, 2100, 70001])
def test_not_finite(heads, buckets, positions, dtype):
    """Infinities of one sign, of both, and NaN reach their own bucket and head; all other sums are as without them."""
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    batch = max(2, 3000 // positions)
    gen = torch.Generator().manual_seed(positions + heads)
    edges = training.distance_edges(buckets, 40)
    announce("not finite %d x %d, %d heads, %d buckets, %s" % (batch, positions, heads, buckets, dtype))
    d = torch.rand((batch, positions), generator=gen) * 60
    up = torch.randn((batch, heads, positions), generator=gen)
    bucket = ref.buckets(d.numpy(), edges.numpy())
    inf, nan = float("inf"), float("nan")
    for h in range(heads):
        odd = [[inf], [inf, -inf], [nan], [-inf, -inf], [inf, nan]][h % 5]
        for value in odd:
            b, p = (int(torch.randint(0, n, (1,), generator=gen)) for n in (batch, positions))
            up[b, h, p] = value
    # opposite infinities in one bucket
    up[0, 0, 0], up[1, 0, positions - 1] = inf, -inf
    d[1, positions - 1] = d[0, 0]
    bucket = ref.buckets(d.numpy(), edges.numpy())
    up = up.to(getattr(torch, TYPES[dtype]))
    got = field_gradient(d.to(dev), edges.to(dev), up.to(dev), heads)
    total, _, _ = ref.gradient(up.double().numpy(), bucket, buckets)
    finite = torch.where(torch.isfinite(up), up, torch.zeros_like(up))
    size = ref.gradient(finite.double().numpy(), bucket, buckets)[1]
    ref.check(got, total, 16 * U * size, "f32", "not finite")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest(dtype):
    """Gradients next to the type's largest whose sums stay in range."""
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    edges = training.distance_edges(20, 40)
    gen = torch.Generator().manual_seed(2)
    d = torch.rand((3, 4000), generator=gen) * 40
    up = torch.randn((3, 5, 4000), generator=gen)
    kind = getattr(torch, TYPES[dtype])
    up[0, 1, 17], up[2, 1, 40], up[1, 3, 3999] = 0.75 * torch.finfo(kind).max, 1e-3, -torch.finfo(kind).max
    d[2, 40] = d[0, 17] + 20 if d[0, 17] < 20 else d[0, 17] - 20
    up = up.to(kind)
    announce("the largest gradients %s" % dtype)
    got = field_gradient(d.to(dev), edges.to(dev), up.to(dev), 5)
    total, size, _ = ref.gradient(up.double().numpy(), ref.buckets(d.numpy(), edges.numpy()), 20)
    assert np.isfinite(got).all()
    ref.check(got, total, 16 * U * size, "f32", "largest")


def test_infinities_cost_little():
    """An infinity in every head, as a scaled loss that overflowed leaves them: the sums are made twice, and
    32 times the time of a clean call is far out."""
    import torch
    from paper_2608_24738_amd import training
    dev = "cuda:0"
    edges = training.distance_edges(32, 1024, signed=True).to(dev)
    up = torch.randn((2, 16, 1024, 1024), device=dev).to(torch.bfloat16)
    table = torch.zeros((32, 16), device=dev, requires_grad=True)
    announce("an infinity in every head")

    def once(up):
        bias = training.relative_bias(table, edges, 1024, 1024, metric="offset", add=up)
        torch.cuda.synchronize()
        begin = time.perf_counter()
        grad, = torch.autograd.grad([bias], [table], [up])
        torch.cuda.synchronize()
        return time.perf_counter() - begin, grad
    clean = sorted(once(up)[0] for _ in range(7))[3]
    up[1, :, 700, 3] = float("inf")
    times, grad = zip(*[once(up) for _ in range(7)])
    print("clean %.0f us, with infinities %.0f us" % (1e6 * clean, 1e6 * sorted(times)[3]), flush=True)
    assert int(torch.isinf(grad[0]).sum()) == 16 and not torch.isnan(grad[0]).any()
    assert sorted(times)[3] < 32 * clean
