"""One gradient alone where the weights cannot be read in place, over the sizes at which g goes from single waves to tiles."""
import pytest

import head_reference as ref
from gpu_util import announce
from test_gpu_head import make, numbers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,d", [(20, 300, 127), (70, 1500, 1003), (130, 700, 515), (300, 513, 511), (300, 3001, 515),
                                   (64, 20001, 250), (1100, 60, 255)])
def test_one_gradient_alone(dtype, n, v, d):
    import torch
    from paper_2608_24738_amd import training
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=11)
    want = ref.exact(numbers(hidden), numbers(weight), labels.cpu().numpy(), 1.0, dtype, (numbers(ups[0]), None), False)
    for which in (0, 1):
        announce("one gradient %s %dx%dx%d %d" % (dtype, n, v, d, which))
        leaves = [hidden.detach().clone(), weight.detach().clone()]
        leaves[which].requires_grad_()
        grad, = torch.autograd.grad(training.head_log_probs(*leaves, labels).log_probs, leaves[which], ups[0])
        ref.check(numbers(grad), want[("dh", "dw")[which]], want[("tol_dh", "tol_dw")[which]], "gradient", dtype)
