"""More rows than there are workgroups for them."""
import pytest

from gpu_util import announce

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,width", [("bfloat16", 32777), ("float32", 16385)])
def test_norm_of_many_long_rows(dtype, width):
    """Rows that no workgroup holds, more of them than 2048 workgroups: each as it is by itself."""
    import torch
    from paper_2608_24738_amd import training
    rows = 2048 + 53
    announce("layer_norm %d x %d %s" % (rows, width, dtype))
    gen = torch.Generator(device="cuda").manual_seed(0)
    t = getattr(torch, dtype)
    x = torch.randn((rows, width), generator=gen, device="cuda").to(t).requires_grad_()
    w = torch.randn(width, generator=gen, device="cuda")
    up = torch.randn((rows, width), generator=gen, device="cuda").to(t)
    y = training.layer_norm(x, w)
    dx, = torch.autograd.grad(y, x, up)
    for part in (slice(0, 60), slice(2040, rows)):
        few = x.detach()[part].requires_grad_()
        want = training.layer_norm(few, w)
        assert torch.equal(y[part], want) and torch.equal(dx[part], torch.autograd.grad(want, few, up[part])[0])
    assert y.isfinite().all() and dx.isfinite().all()


def test_gradient_of_a_table_of_2_30_rows():
    """A workgroup to 64 rows, of which the grid's first axis has eight threads."""
    import torch
    from paper_2608_24738_amd import training
    rows = (1 << 30) + 70
    announce("embedding's gradient, %d rows of 1" % rows)
    table = torch.zeros((rows, 1), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    tokens = torch.tensor([0, 1, 64, 12345678, 1 << 29, (1 << 30) - 1, 1 << 30, rows - 1, rows, -1, 64], device="cuda")
    up = torch.arange(1, 12, device="cuda").bfloat16()[:, None]
    grad, = torch.autograd.grad(training.embedding(tokens, table), table, up)
    assert int(torch.count_nonzero(grad)) == 8
    assert grad[tokens[:8], 0].tolist() == [1, 2, 3 + 11, 4, 5, 6, 7, 8]
