"""Layer norm and its gradients against float64.

Bounds, with u = 2^-24: a float32 sum of n terms is off by at most u (8 + 4 sqrt n) times the sum of their sizes (the
additions' roundings add up like a random walk, for which that is far out).  What follows is carried through the
formulas to first order, with a few u for each operation.
"""
import numpy as np
import pytest

from gpu_util import announce
from head_reference import U, check, walk

pytestmark = pytest.mark.gpu

KINDS = {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}


def exact(x, w, b, eps, g):
    n, d = x.shape
    eps = float(np.float32(eps))
    m = x.mean(1, keepdims=True)
    v = x - m
    var = (v * v).mean(1, keepdims=True)
    r = 1 / np.sqrt(var + eps)
    t = v * r
    em = walk(d) * np.abs(x).mean(1, keepdims=True) + U * np.abs(m)
    ev = em + U * np.abs(v)
    # sum v em = 0 but for em's square; the rest of var is relative
    er = 0.5 * (walk(d) + 4 * U + em * em * r * r) + 4 * U
    et = ev * r + np.abs(t) * (er + 2 * U)
    out = {"y": t * w + b}
    out["tol_y"] = np.abs(w) * et + 2 * U * (np.abs(t * w) + np.abs(b))
    gw = g * w
    a, c = gw.mean(1, keepdims=True), (gw * t).mean(1, keepdims=True)
    ea = walk(d) * np.abs(gw).mean(1, keepdims=True) + 2 * U * np.abs(a)
    ec = walk(d) * np.abs(gw * t).mean(1, keepdims=True) + (np.abs(gw) * et).mean(1, keepdims=True) + 2 * U * np.abs(c)
    out["dx"] = r * (gw - a - t * c)
    out["tol_dx"] = r * (ea + np.abs(t) * ec + et * np.abs(c) + 4 * U * (np.abs(gw) + np.abs(a) + np.abs(t * c))) \
        + np.abs(out["dx"]) * (er + 2 * U)
    out["dw"], out["db"] = (g * t).sum(0), g.sum(0)
    out["tol_dw"] = (np.abs(g) * et).sum(0) + walk(n) * np.abs(g * t).sum(0)
    out["tol_db"] = walk(n) * np.abs(g).sum(0)
    return out


def make(n, d, dtype, affine, pad=0, shift=0, offset=0.0, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed + 31 * n + d)
    kind = getattr(torch, KINDS[dtype])
    flat = torch.full((shift + n * (d + pad),), float("nan"), dtype=kind, device="cuda")
    x = flat[shift:].view(n, d + pad)[:, :d]
    x.copy_((torch.randn(n, d, generator=gen) * (0.5 + torch.rand(n, 1, generator=gen)) + offset).to(kind))
    w = b = None
    if affine:
        w = (1 + 0.3 * torch.randn(d, generator=gen)).to(getattr(torch, KINDS[affine])).cuda()
        b = torch.randn(d, generator=gen).to(w.dtype).cuda()
    up = torch.randn(n, d, generator=gen).to(kind).cuda()
    return x, w, b, up


def numbers(t):
    return t.detach().double().cpu().numpy()


def run(x, w, b, up, eps=1e-5):
    import torch
    from paper_2608_24738_amd import training
    leaves = [t.detach().requires_grad_() for t in (x, w, b) if t is not None]
    rest = iter(leaves[1:])
    out = training.layer_norm(leaves[0], None if w is None else next(rest), None if b is None else next(rest), eps=eps)
    grads = torch.autograd.grad(out, leaves, up)
    torch.cuda.synchronize()
    return out, grads


def compare(x, w, b, up, dtype, affine, what, eps=1e-5):
    announce(what)
    out, grads = run(x, w, b, up, eps)
    d = x.shape[1]
    want = exact(numbers(x), np.ones(d) if w is None else numbers(w), np.zeros(d) if b is None else numbers(b), eps,
                 numbers(up))
    check(numbers(out), want["y"], want["tol_y"], "y", dtype)
    check(numbers(grads[0]), want["dx"], want["tol_dx"], "dx", dtype)
    names = [name for name, t in (("dw", w), ("db", b)) if t is not None]
    for grad, name in zip(grads[1:], names):
        check(numbers(grad), want[name], want["tol_" + name], name, affine)
    assert out.dtype == x.dtype and all(g.dtype == t.dtype for g, t in zip(grads, [t for t in (x, w, b) if t is not None]))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,d", [
    (1, 1), (3, 1), (1, 2), (5, 7), (17, 16), (33, 64), (70, 100), (4, 127), (9, 200), (20, 257), (2, 512), (40, 1000),
    (3, 1024), (19, 2048), (5, 2500), (3, 4096), (7, 4099), (2, 8192), (3, 9001), (2, 16384), (3, 20000), (2, 33001),
    (1, 40000), (1000, 24), (3000, 333)])
def test_sizes(dtype, n, d):
    compare(*make(n, d, dtype, "f32"), dtype, "f32", "norm %s %dx%d" % (dtype, n, d))


@pytest.mark.parametrize("dtype,affine", [("bf16", "bf16"), ("f16", "f16"), ("bf16", None), ("f32", None), ("f32", "bf16"),
                                          ("f16", "f32")])
@pytest.mark.parametrize("n,d", [(6, 65), (50, 768), (3, 5000), (2, 40001)])
def test_parameter_types(dtype, affine, n, d):
    compare(*make(n, d, dtype, affine), dtype, affine, "norm params %s %s %dx%d" % (dtype, affine, n, d))


@pytest.mark.parametrize("n,d,pad,shift", [(5, 64, 1, 0), (5, 64, 8, 1), (7, 1001, 23, 3), (3, 4097, 3, 1), (2, 35000, 1, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype, n, d, pad, shift):
    """Rows that are parts of longer ones, beside which lies NaN."""
    compare(*make(n, d, dtype, "f32", pad=pad, shift=shift), dtype, "f32", "norm strides %s" % ((dtype, n, d, pad, shift),))


@pytest.mark.parametrize("d", [48, 1000, 6000, 40000])
def test_rows_far_from_zero(d):
    """A mean of 1000 deviations: what the squares are taken of has lost nothing."""
    compare(*make(5, d, "f32", "f32", offset=1000.0), "f32", "f32", "norm offset %d" % d)


def test_weight_or_bias_alone():
    import torch
    x, w, b, up = make(30, 300, "bf16", "f32")
    compare(x, w, None, up, "bf16", "f32", "norm weight alone")
    compare(x, None, b, up, "bf16", "f32", "norm bias alone")
    from paper_2608_24738_amd import training
    full = run(x, w, b, up)
    for which in range(3):
        leaves = [t.detach().clone() for t in (x, w, b)]
        leaves[which].requires_grad_()
        grad, = torch.autograd.grad(training.layer_norm(*leaves), leaves[which], up)
        assert torch.equal(grad, full[1][which])


@pytest.mark.parametrize("d", [40, 700, 5000, 40000])
def test_rows_that_are_constant_or_not_finite(d):
    import torch
    x, w, b, up = make(6, d, "f32", "f32")
    base = run(x, w, b, up)
    x[1] = 3.0
    out, grads = run(x, w, b, up)
    # a constant row: its mean is off by roundings alone, of which 1 / sqrt(eps) makes some 2^-12
    assert (out[1] - b).abs().max() <= 320 * 3 * walk(d) * (1 + w.abs().max()) and grads[0].isfinite().all()
    x[2, d // 2] = float("nan")
    x[4, 0] = float("inf")
    out, grads = run(x, w, b, up)
    bad = torch.tensor([2, 4], device="cuda")
    good = torch.tensor([0, 3, 5], device="cuda")
    assert out[bad].isnan().all() and grads[0][bad].isnan().all()
    assert torch.equal(out[good], base[0][good]) and torch.equal(grads[0][good], base[1][0][good])


def test_shapes():
    import torch
    from paper_2608_24738_amd import training
    x, w, b, up = make(24, 50, "bf16", "bf16")
    flat = training.layer_norm(x, w, b)
    assert torch.equal(training.layer_norm(x.view(2, 3, 4, 50), w, b).view(24, 50), flat)
    assert torch.equal(training.layer_norm(x[0], w, b), flat[0])
    turned = x.view(4, 6, 50).transpose(0, 1)
    assert torch.equal(training.layer_norm(turned, w, b), flat.view(4, 6, 50).transpose(0, 1))
    assert torch.equal(training.layer_norm(x.t().contiguous().t(), w, b), flat)
    row = x[:1].detach().requires_grad_()
    wide = training.layer_norm(row.expand(24, 50), w, b)
    assert torch.equal(wide, flat[:1].expand(24, 50))
    wide.sum().backward()
    assert row.grad.shape == row.shape
    leaf = w.detach().requires_grad_()
    none = training.layer_norm(x[:0], leaf, b)
    assert none.shape == (0, 50)
    none.sum().backward()
    assert not leaf.grad.any()


def test_difference_quotients():
    import torch
    x, w, b, up = make(5, 37, "f32", "f32")
    grads = [g.double().cpu() for g in run(x, w, b, up)[1]]
    base = [t.double().cpu() for t in (x, w, b)]
    up = up.double().cpu()

    def value(x, w, b):
        v = x - x.mean(1, keepdim=True)
        return (up * (v / ((v * v).mean(1, keepdim=True) + float(np.float32(1e-5))).sqrt() * w + b)).sum()
    gen = torch.Generator().manual_seed(3)
    for _ in range(4):
        e = [torch.randn(t.shape, generator=gen).double() for t in base]
        step = 1e-5
        slope = (value(*[t + step * d for t, d in zip(base, e)]) - value(*[t - step * d for t, d in zip(base, e)])) / (2 * step)
        have = sum((g * d).sum() for g, d in zip(grads, e))
        size = sum((g * d).abs().sum() for g, d in zip(grads, e))
        # float32 gradients are off by some 100 u of their sizes, the quotient by 1e-10 of third derivatives
        assert abs(slope - have) <= 2.0 ** -17 * size + 1e-7


def test_two_calls_give_the_same_bits_and_replays_too():
    import torch
    from paper_2608_24738_amd import training
    x, w, b, up = make(3000, 520, "bf16", "f32")
    x = x.contiguous()
    a, c = run(x, w, b, up), run(x, w, b, up)
    assert torch.equal(a[0], c[0]) and all(torch.equal(p, q) for p, q in zip(a[1], c[1]))
    leaves = [t.detach().clone().requires_grad_() for t in (x, w, b)]

    def step():
        out = training.layer_norm(*leaves)
        return (out,) + torch.autograd.grad(out, leaves, up)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        new = make(3000, 520, "bf16", "f32", seed=i + 1)
        with torch.no_grad():
            for leaf, t in zip(leaves, new):
                leaf.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.detach().clone() for t in out]
        eager = run(*leaves, up)
        for p, q in zip(kept, [eager[0]] + list(eager[1])):
            assert torch.equal(p, q)
