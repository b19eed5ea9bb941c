"""Layer norm of rows that lie far from zero: what is left of the mean's own rounding.

With u = 2^-24 and W = walk(width) the relative error that a float32 sum may have: the first mean is off by c W for rows
around c, the differences from it are exact (or off by half a step of theirs), and so is what their mean is off by, up to
W of that.  The result is therefore off by c W^2 r, beside the roundings of the formula on t, the result itself, which are
those of differences, squares, their sum, the root and the product: 8 u + W.
"""
import numpy as np
import pytest

import head_reference as ref
from gpu_util import announce

pytestmark = pytest.mark.gpu

WIDTHS = [3, 17, 64, 100, 255, 1000, 1001, 3001, 5000, 16384, 40001, 70000]


def case(rows, width, dtype, centre, spread, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = centre + spread * torch.randn(rows, width, generator=gen, dtype=torch.float64)
    return x.to(getattr(torch, dtype)).cuda()


def check(x, eps=1e-5):
    from paper_2608_24738_amd import training
    y = training.layer_norm(x, eps=eps).double().cpu().numpy()
    v = x.double().cpu().numpy()
    width = v.shape[1]
    e = float(np.float32(eps))
    m = v.mean(1, keepdims=True)
    r = 1 / np.sqrt(((v - m) ** 2).mean(1, keepdims=True) + e)
    t = (v - m) * r
    w = ref.walk(width)
    size = np.abs(v).mean(1, keepdims=True)
    tol = (8 * ref.U + w) * np.abs(t) + 2 * size * w * w * r
    ref.check(y, t, tol, "norm", {"float32": "f32", "bfloat16": "bf16", "float16": "f16"}[str(x.dtype).split(".")[1]])


@pytest.mark.parametrize("width", WIDTHS)
def test_constant_rows(width):
    """Rows of one number each have nothing left beside their mean."""
    import torch
    announce("constant rows of %d" % width)
    for centre in (0.1, 1000.1, -12345.678, 3.3e6):
        check(case(3, width, "float32", centre, 0.0, 0))
    check(case(3, width, "bfloat16", 300.0, 0.0, 0))
    check(case(3, width, "float16", -1003.0, 0.0, 0))


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("centre,spread", [(1000.0, 0.5), (-20000.0, 3.0), (1.0, 1e-3)])
def test_far_rows(width, centre, spread):
    announce("rows of %d around %g" % (width, centre))
    check(case(3, width, "float32", centre, spread, width))


@pytest.mark.parametrize("width", WIDTHS)
def test_gradient_of_far_rows(width):
    """dx, dw and db take t from the rounded mean that is kept, half a step of it off: t by c u r."""
    import torch
    from paper_2608_24738_amd import training
    announce("gradient of rows of %d" % width)
    x = case(5, width, "float32", 1000.0, 0.5, width).requires_grad_()
    gen = torch.Generator().manual_seed(width)
    w = (1 + 0.1 * torch.randn(width, generator=gen)).cuda().requires_grad_()
    b = torch.zeros(width, device="cuda", requires_grad=True)
    up = torch.randn(5, width, generator=gen).cuda()
    grads = torch.autograd.grad(training.layer_norm(x, w, b), [x, w, b], up)
    v, g, k = (t.detach().double().cpu().numpy() for t in (x, up, w))
    m = v.mean(1, keepdims=True)
    r = 1 / np.sqrt(((v - m) ** 2).mean(1, keepdims=True) + float(np.float32(1e-5)))
    t = (v - m) * r
    walk = ref.walk(width)
    off = (8 * ref.U + walk) * np.abs(t) + (2 * walk * walk + 2 * ref.U) * np.abs(m) * r
    gw = g * k
    mean, along = gw.mean(1, keepdims=True), (gw * t).mean(1, keepdims=True)
    size, size_t = np.abs(gw).mean(1, keepdims=True), np.abs(gw * t).mean(1, keepdims=True)
    off_along = (np.abs(gw) * off).mean(1, keepdims=True) + walk * size_t
    want = r * (gw - mean - t * along)
    tol = r * (walk * size + off * np.abs(along) + np.abs(t) * off_along + off * off_along
               + (12 * ref.U + walk) * (np.abs(gw) + np.abs(mean) + np.abs(t * along)))
    ref.check(grads[0].double().cpu().numpy(), want, tol, "dx")
    ref.check(grads[1].double().cpu().numpy(), (g * t).sum(0), (np.abs(g) * off).sum(0) + ref.walk(5) * np.abs(g * t).sum(0), "dw")
    ref.check(grads[2].double().cpu().numpy(), g.sum(0), ref.walk(5) * np.abs(g).sum(0), "db")
