"""Forward-mode derivatives are refused, as second derivatives are: a call would return values without their tangents."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2608_24738_amd import training


def test_tangents_are_seen():
    x = torch.zeros(3)
    training._reverse_only(x, None)
    with forward_ad.dual_level():
        training._reverse_only(x, None)
        dual = forward_ad.make_dual(x, torch.ones(3))
        for tensors in ((dual,), (x, dual), (None, dual.reshape(1, 3)), (dual[1:],)):
            with pytest.raises(RuntimeError, match="forward"):
                training._reverse_only(*tensors)
        training._reverse_only(forward_ad.unpack_dual(dual).primal, dual.detach().clone())


@pytest.mark.gpu
def test_refused():
    from gpu_util import announce
    announce("forward-mode derivatives")
    dev = "cuda:0"
    x, y = torch.randn((2, 5, 7), device=dev), torch.zeros((2, 7), dtype=torch.int64, device=dev)
    table, edges = torch.randn((4, 3), device=dev), torch.tensor([1.0, 2.0, 3.0], device=dev)
    d, scores = torch.rand((2, 6), device=dev), torch.randn((2, 3, 5, 5), device=dev)
    extra = torch.randn((2, 3, 6), device=dev)
    calls = [(x, lambda t: training.label_log_probs(t, y)),
             (x, lambda t: training.label_log_probs(t, top_k=1)),
             (x, lambda t: training.label_log_probs(x, y, field=t)),
             (x[:, :, :1], lambda t: training.label_log_probs(x, y, field=t)),
             (table, lambda t: training.relative_bias(t, edges, 5, 5)),
             (table, lambda t: training.distance_bias(d, t, edges)),
             (edges, lambda t: training.distance_bias(d, table, t)),
             (scores, lambda t: training.relative_bias(table, edges, 5, 5, add=t)),
             (extra, lambda t: training.distance_bias(d, table, edges, add=t)),
             (d, lambda t: training.distance_bias(t, table, edges))]
    for t, call in calls:
        call(t)
        with forward_ad.dual_level():
            call(t)
            dual = forward_ad.make_dual(t.detach(), torch.ones_like(t))
            with pytest.raises(RuntimeError, match="forward"):
                call(dual)
            with pytest.raises(RuntimeError), torch.no_grad():
                call(dual)
        with pytest.raises(RuntimeError):
            torch.func.jvp(lambda z: call(z), (t,), (torch.ones_like(t),))
    torch.cuda.synchronize()
