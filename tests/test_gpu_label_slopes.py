"""Gradients of label_log_probs that are very small, against the definitions in float64."""
import numpy as np
import pytest

import label_reference as ref
from gpu_util import announce
from test_gpu_labels import case

pytestmark = pytest.mark.gpu


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
