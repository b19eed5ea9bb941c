"""Gradients of label_log_probs in which terms cancel or are very small, against the definitions in float64."""
import numpy as np
import pytest

import label_reference as ref
from gpu_util import announce
from test_gpu_labels import TYPES, case, run

pytestmark = pytest.mark.gpu

# Each of the kernels: held classes, running ones, short rows, rows by waves, rows with rounds against a reference.
SHAPES = [(50, 2), (3, 2, 70), (2, 21, 60), (2, 30, 41), (3, 40, 50), (40, 64), (4100, 100), (9, 700), (5, 5000),
          (2050, 4600)]


def lifted(shape, dtype, offset, seed):
    """Logits around `offset` whose label is the likeliest class by 4 to 20, as far as the type tells them apart."""
    import torch
    x, _, _, ups = case(shape, "f32", seed=seed, scale=0.5)
    gen = torch.Generator().manual_seed(seed)
    rest = shape[:1] + shape[2:]
    y = torch.randint(0, shape[1], rest, generator=gen).to(x.device)
    gap = (4 + 16 * torch.rand(rest, generator=gen)).to(x.device) + np.log(shape[1])
    x = x.scatter_add(1, y[:, None], gap[:, None]) + offset
    return x.to(getattr(torch, TYPES[dtype])), y, ups


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("offset", [0.0, 15.0, 50.0, 120.0, -120.0, 517.0, -904.0, 960.0])
@pytest.mark.parametrize("shape", SHAPES)
def test_likely_labels(shape, offset, dtype):
    """The slope of a likely label is what is left of 1 - p."""
    x, y, ups = lifted(shape, dtype, offset, seed=int(abs(offset)) + shape[1])
    run(x, y, ups=[ups[0], None, None], what="likely labels around %g %s" % (offset, dtype), dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("offset", [0.0, 60.0, 130.5, 523.0, 777.5, -777.5, 960.0])
@pytest.mark.parametrize("where", ["map", "row"])
def test_two_classes(offset, dtype, where):
    """Two classes, the label's ahead by 0 to 16.  With u = 2^-24: the sum of exponentials 1 + e is off by u and what
    e is off by, its logarithm by 4 u of itself and u, the exponent of p by u of itself (below 1 here) and what the
    parts of m + log s that were rounded away leave in second order (below 0.1 u), the exponential by 4 u, the
    products behind it by 1 u each: 16 u of the upstream gradient in all."""
    import torch
    from paper_2608_24738_amd import training
    kind = getattr(torch, TYPES[dtype])
    gap = torch.linspace(0, 16, 257)
    x = torch.stack([gap.clone(), torch.zeros(257)], 1 if where == "row" else 0) + offset
    x = (x[None] if where == "map" else x).to(kind).to("cuda:0")
    y = torch.zeros((1, 257) if where == "map" else (257,), dtype=torch.int64, device=x.device)
    announce("two classes around %g %s %s" % (offset, dtype, where))
    x.requires_grad_(True)
    grad, = torch.autograd.grad([training.label_log_probs(x, y).log_probs], [x], [torch.ones(y.shape, device=x.device)])
    z = x.detach().double().cpu().numpy()
    z = z if where == "row" else z[0].T
    # 1 - p of the label's class, without cancellation
    rest = 1.0 / (1.0 + np.exp(z[:, 0] - z[:, 1]))
    want = np.stack([rest, -rest], 1)
    got = grad.double().cpu().numpy()
    ref.check(got if where == "row" else got[0].T, want, 16 * ref.U, "gradient", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("offset", [50.0, 130.5, -523.0, 960.0])
@pytest.mark.parametrize("shape", SHAPES)
def test_equal_logits(shape, offset, dtype):
    """All classes alike: the entropy is at its largest and has no slope, the field's mean one by the field alone."""
    import torch
    x, y, phi, ups = case(shape, dtype, seed=3, field=True)
    x = torch.full_like(x, offset)
    run(x, y, field=phi, ups=[None, ups[1], None], what="entropy of equal logits " + dtype, dtype=dtype)
    run(x, y, field=phi, ups=ups, what="equal logits " + dtype, dtype=dtype)


@pytest.mark.parametrize("scale", [1e-30, 1e-34, 1e-36, 1e30])
@pytest.mark.parametrize("shape", [(3, 4, 50), (3, 40, 50), (5, 700), (4100, 100)])
def test_small_upstream(shape, scale):
    """Upstream gradients far from 1, down to float32's smallest: the logits' are theirs times ordinary factors.
    Products may fall among float32's subnormals, 2^-149 apart: four of them to a gradient."""
    import torch
    from paper_2608_24738_amd import training
    x, y, phi, ups = case(shape, "f32", seed=6, field=True, scale=1.0)
    small = [u * scale for u in ups]
    announce("upstream gradients of %g, logits %s" % (scale, shape))
    x.requires_grad_(True)
    got = training.label_log_probs(x, y, entropy=True, field=phi)
    grad, = torch.autograd.grad([got.log_probs, got.entropy, got.field_mean], [x], small)
    flat = lambda t: t.detach().movedim(1, -1).reshape(-1, shape[1]).double().cpu().numpy()
    want = ref.exact(flat(x), y.reshape(-1).cpu().numpy(), flat(phi), 0,
                     [u.double().cpu().numpy().reshape(-1) / scale for u in small])
    ref.check(flat(grad) / scale, want["grad"], want["tol_grad"] + 4 * 2.0 ** -149 * (1 + np.abs(flat(phi))) / scale,
              "gradient")
