"""Rows of a table by given tokens, and the table's gradient, against float64.

The lookup is one product and one rounding, which torch does alike.  A row of the gradient is a float32 sum of its n
terms, off by at most u (8 + 4 sqrt n) of the sum of their sizes, times the scale, rounded once.
"""
import numpy as np
import pytest

from gpu_util import announce
from head_reference import U, check, walk

pytestmark = pytest.mark.gpu

KINDS = {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}


def make(tokens, rows, width, dtype, how="zipf", kind="int64", seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed + 7 * tokens + 3 * rows + width)
    if how == "same":
        k = torch.full((tokens,), rows // 2)
    elif how == "outside":
        k = torch.where(torch.rand(tokens, generator=gen) < 0.5, torch.full((tokens,), -1), torch.full((tokens,), rows))
    elif how == "ends":
        k = torch.where(torch.rand(tokens, generator=gen) < 0.5, torch.zeros(tokens, dtype=torch.int64), torch.full((tokens,), rows - 1))
    elif how == "falling":
        k = torch.arange(tokens - 1, -1, -1) % rows
    else:
        k = (rows * torch.rand(tokens, generator=gen) ** 4).long().clamp_max(rows - 1)
        lost = torch.rand(tokens, generator=gen) < 0.1
        k = torch.where(lost, torch.tensor([-1, rows, rows + 5, -100])[torch.arange(tokens) % 4], k)
    if kind == "uint8":
        k = torch.where((k < 0) | (k > 255), torch.full_like(k, 255), k)
    t = getattr(torch, KINDS[dtype])
    table = torch.randn(rows, width, generator=gen).to(t).cuda()
    up = torch.randn(tokens, width, generator=gen).to(t).cuda()
    return k.to(getattr(torch, kind)).cuda(), table, up


def run(tokens, table, up, scale):
    import torch
    from paper_2608_24738_amd import training
    leaf = table.detach().requires_grad_()
    out = training.embedding(tokens, leaf, scale=scale)
    grad, = torch.autograd.grad(out, leaf, up)
    torch.cuda.synchronize()
    return out, grad


def numbers(t):
    return t.detach().double().cpu().numpy()


def compare(tokens, table, up, scale, dtype, what):
    import torch
    announce(what)
    out, grad = run(tokens, table, up, scale)
    k = tokens.long().cpu().numpy().reshape(-1)
    rows, width = table.shape
    real = (k >= 0) & (k < rows)
    look = torch.zeros(len(k), width, device="cuda")
    index = torch.from_numpy(np.flatnonzero(real)).cuda()
    look[index] = table.float()[torch.from_numpy(k[real]).cuda()] * scale
    assert torch.equal(out.reshape(-1, width), look.to(table.dtype))
    g = numbers(up).reshape(-1, width)
    want, size, count = np.zeros((rows, width)), np.zeros((rows, width)), np.zeros(rows)
    np.add.at(want, k[real], g[real])
    np.add.at(size, k[real], np.abs(g[real]))
    np.add.at(count, k[real], 1)
    scale = float(np.float32(scale))
    check(numbers(grad), scale * want, abs(scale) * (walk(count)[:, None] * size + U * np.abs(want)), "grad", dtype)
    return out, grad


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,rows,width", [
    (1, 1, 1), (1, 100, 64), (2, 7, 8), (15, 3, 5), (16, 300, 33), (17, 2, 128), (100, 50, 257), (1000, 255, 40),
    (2048, 511, 16), (2049, 512, 24), (5000, 70000, 9), (4097, 131, 1030), (9000, 1 << 18, 4), (300, 20, 4100)])
def test_sizes(dtype, tokens, rows, width):
    compare(*make(tokens, rows, width, dtype), 1.0, dtype, "embedding %s %d of %dx%d" % (dtype, tokens, rows, width))


@pytest.mark.parametrize("how", ["same", "outside", "ends", "falling"])
@pytest.mark.parametrize("tokens,rows,width", [(1, 9, 16), (40, 9, 16), (16, 4, 100), (5001, 90, 72), (4096, 1000, 520)])
def test_orders(how, tokens, rows, width):
    compare(*make(tokens, rows, width, "bf16", how), 2.5, "bf16", "embedding %s %d of %dx%d" % (how, tokens, rows, width))


@pytest.mark.parametrize("scale", [0.0, -0.3, 32.0, 1e-3])
def test_scales(scale):
    compare(*make(200, 30, 50, "f16"), scale, "f16", "embedding scale %s" % scale)


@pytest.mark.parametrize("kind", ["uint8", "int32", "int64"])
def test_token_types(kind):
    compare(*make(500, 200, 24, "f32", kind=kind), 1.0, "f32", "embedding tokens %s" % kind)


@pytest.mark.parametrize("tokens,how", [(150001, "zipf"), (200000, "same"), (140000, "falling")])
def test_many_tokens(tokens, how):
    """More tiles than a workgroup adds up by itself, longer chunks, rows over many of them."""
    compare(*make(tokens, 1500, 12, "bf16", how), 1.0, "bf16", "embedding many %d %s" % (tokens, how))


@pytest.mark.parametrize("kind", ["int32", "int64"])
@pytest.mark.parametrize("tokens,rows,how", [
    (32768, 20011, "zipf"), (32769, 20011, "zipf"), (32768, 700, "same"), (30000, 511, "outside"), (17000, 131072, "falling"),
    (1025, 65536, "same"), (9000, (1 << 19) - 1, "outside"), (9000, 1 << 19, "outside"), (16383, 2, "falling")])
def test_sorted_by_ranges_and_by_digits(tokens, rows, how, kind):
    """The most tokens and rows of a workgroup to a range of rows, one more of each, and all tokens in one range."""
    compare(*make(tokens, rows, 3, "f32", how, kind), 1.0, "f32", "embedding %s %s %d of %d" % (kind, how, tokens, rows))


def test_shapes_strides_and_no_tokens():
    import torch
    from paper_2608_24738_amd import training
    tokens, table, up = make(60, 40, 24, "bf16")
    flat, grad = run(tokens, table, up, 1.0)
    many, same = run(tokens.view(3, 4, 5), table, up.view(3, 4, 5, 24), 1.0)
    assert torch.equal(many.view(60, 24), flat) and torch.equal(same, grad)
    wide = torch.full((40, 31), float("nan"), dtype=table.dtype, device="cuda")
    wide[:, 3:27] = table
    assert torch.equal(training.embedding(tokens, wide[:, 3:27]), flat)
    assert torch.equal(training.embedding(tokens, table.t().contiguous().t()), flat)
    every = torch.empty(120, dtype=torch.int64, device="cuda")
    every[::2] = tokens
    assert torch.equal(training.embedding(every[::2], table), flat)
    spread = torch.empty(60, 48, dtype=table.dtype, device="cuda")
    spread[:, ::2] = up
    assert torch.equal(run(tokens, table, spread[:, ::2], 1.0)[1], grad)
    one = training.embedding(tokens[0], table)
    assert torch.equal(one, flat[0])
    out, none = run(tokens[:0], table, up[:0], 1.0)
    assert out.shape == (0, 24) and none.shape == table.shape and not none.any()


def test_values_that_are_not_finite():
    """An infinity or NaN reaches its own row alone, and one of a token outside the table none."""
    import torch
    tokens, table, up = make(3000, 90, 20, "f32")
    k = tokens.long()
    _, base = run(tokens, table, up, 1.0)
    lost = ((k < 0) | (k >= 90)).nonzero()[:, 0]
    up[lost] = float("nan")
    _, got = run(tokens, table, up, 1.0)
    assert torch.equal(got, base)
    up[(k == 0).nonzero()[5]] = float("nan")
    up[(k == 7).nonzero()[0]] = float("inf")
    _, got = run(tokens, table, up, 1.0)
    assert got[0].isnan().all() and (got[7] == float("inf")).all()
    keep = torch.ones(90, dtype=torch.bool, device="cuda")
    keep[0] = keep[7] = False
    assert torch.equal(got[keep], base[keep])


def test_difference_quotients():
    import torch
    tokens, table, up = make(90, 12, 10, "f32")
    _, grad = run(tokens, table, up, 0.7)
    k, t, g = tokens.cpu(), table.double().cpu(), up.double().cpu()
    real = (k >= 0) & (k < 12)

    def value(t):
        return (g[real] * float(np.float32(0.7)) * t[k[real]]).sum()
    e = torch.randn(t.shape, generator=torch.Generator().manual_seed(1)).double()
    slope = (value(t + 1e-3 * e) - value(t - 1e-3 * e)) / 2e-3
    have = (grad.double().cpu() * e).sum()
    # linear: the quotient has rounding alone
    assert abs(slope - have) <= 2.0 ** -18 * (grad.double().cpu() * e).abs().sum() + 1e-9


def test_two_calls_give_the_same_bits_and_replays_too():
    import torch
    from paper_2608_24738_amd import training
    tokens, table, up = make(20000, 700, 136, "bf16")
    a, b = run(tokens, table, up, 1.0), run(tokens, table, up, 1.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    leaf = table.detach().clone().requires_grad_()

    def step():
        out = training.embedding(tokens, leaf)
        return (out,) + torch.autograd.grad(out, leaf, up)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        tokens.copy_(make(20000, 700, 136, "bf16", seed=i + 1)[0])
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.detach().clone() for t in out]
        eager = run(tokens, leaf, up, 1.0)
        assert torch.equal(kept[0], eager[0]) and torch.equal(kept[1], eager[1])
