"""Rows with a NaN or +inf among rows without: every float of those is NaN, and of no others."""
import pytest

from gpu_util import announce
from test_gpu_labels import TYPES, case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("shape", [(4099, 33), (4099, 100), (4099, 256), (4099, 513), (40, 700), (9, 5000), (2, 70001),
                                   (40, 2), (3, 21, 40), (3, 40, 50)])
def test_their_own(shape, dtype):
    import torch
    from paper_2608_24738_amd import training
    x, y, phi, ups = case(shape, dtype, seed=shape[1], field=True, spread_labels=False)
    announce("not finite, logits %s %s" % (shape, dtype))
    rest = (0,) * (x.dim() - 2)
    bad = torch.zeros(y.shape, dtype=torch.bool, device=x.device)
    x[(0, shape[1] - 1) + rest] = torch.nan
    x[(1, 1) + rest] = torch.inf
    bad[(0,) + rest] = bad[(1,) + rest] = True
    k = min(shape[1], 3)

    def call(x, *wants):
        x = x.detach().requires_grad_(True)
        got = training.label_log_probs(x, y, **dict(wants))
        outs = [t for t in got[:3] if t is not None]
        return got, outs, torch.autograd.grad(outs, [x], ups[:len(outs)])[0]
    for wants in ((), (("entropy", True),), (("entropy", True), ("field", phi)), (("top_k", k),)):
        got, outs, grad = call(x, *wants)
        for t in outs:
            assert torch.isnan(t[bad]).all() and torch.isfinite(t[~bad]).all()
        assert torch.isnan(grad.movedim(1, -1)[bad]).all() and torch.isfinite(grad.movedim(1, -1)[~bad]).all()
        if got.top_indices is not None:
            assert ((got.top_indices >= 0) & (got.top_indices < shape[1])).all()
            assert torch.isfinite(got.top_log_probs.movedim(1, -1)[~bad]).all()
    # without a label the log-probability is 0 all the same
    none = training.label_log_probs(x, torch.full_like(y, -1), entropy=True)
    assert not none.log_probs.any() and torch.isnan(none.entropy[bad]).all()
