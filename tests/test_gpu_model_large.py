"""The operators around a vocabulary where offsets pass 2^32 bytes or elements, at a few places against float64."""
import numpy as np
import pytest

import head_reference as ref
from gpu_util import announce

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [3, 40])
def test_large_weight(n):
    """A weight of 4.9e9 elements.  Its far rows decide: the labels are there, and so is most of the mass."""
    import torch
    from paper_2608_24738_amd import training
    v, d = 300011, 16384
    announce("head_log_probs %d x %d x %d bf16" % (n, v, d))
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = torch.empty((v, d), dtype=torch.bfloat16, device="cuda").uniform_(-0.02, 0.02, generator=gen)
    y = torch.randint(v - 1000, v, (n,), generator=gen, device="cuda")
    h = torch.randn((n, d), generator=gen, device="cuda").add_(8 * w[y].float()).bfloat16()
    up = torch.randn(n, generator=gen, device="cuda")
    leaves = [h.requires_grad_(), w.requires_grad_()]
    got = training.head_log_probs(*leaves, y)
    dh, dw = torch.autograd.grad(got.log_probs, leaves, up)
    with torch.no_grad():
        x = torch.cat([h.double() @ w[i:i + 20000].double().t() for i in range(0, v, 20000)], 1)
        total = torch.logsumexp(x, 1)
        want = x.gather(1, y[:, None])[:, 0] - total
        size = float((h.double().abs() @ w[y].double().abs().t()).max())
        off = 2 * ref.walk(d) * size + 2 * ref.U * float(x.abs().max()) + ref.walk(v, 8)
        assert (got.log_probs.double() - want).abs().max() <= off + 4 * ref.U * float(want.abs().max())
        g = -up[:, None].double() * (x - total[:, None]).exp()
        g[torch.arange(n), y] += up.double()
        # slopes are off by `off` relatively, or by half a step of two bf16 numbers, which is less
        tol = (off + 2.0 ** -16) * g.abs()
        for rows in (slice(0, 3), slice(v // 2, v // 2 + 3), slice(v - 1000, v)):
            hd = h.double()
            exact, room = g[:, rows].t() @ hd, tol[:, rows].t() @ hd.abs() + ref.walk(n) * (g[:, rows].abs().t() @ hd.abs())
            ref.check(dw[rows].double().cpu(), exact.cpu(), room.cpu().numpy(), "weight's gradient", "bf16")
        exact = torch.zeros((n, d), dtype=torch.float64, device="cuda")
        room = torch.zeros_like(exact)
        for i in range(0, v, 20000):
            part = w[i:i + 20000].double()
            exact += g[:, i:i + 20000] @ part
            room += (tol[:, i:i + 20000] + ref.walk(v) * g[:, i:i + 20000].abs()) @ part.abs()
        ref.check(dh.double().cpu(), exact.cpu(), room.cpu().numpy(), "hidden's gradient", "bf16")


def test_large_norm():
    import torch
    from paper_2608_24738_amd import training
    n, d = 300007, 16384
    announce("layer_norm %d x %d bf16" % (n, d))
    x = torch.empty((n, d), dtype=torch.bfloat16, device="cuda").uniform_(-4, 4)
    w = torch.linspace(0.5, 1.5, d, device="cuda").requires_grad_()
    x.requires_grad_()
    out = training.layer_norm(x, w)
    up = torch.empty_like(out).uniform_(-1, 1)
    dx, dw = torch.autograd.grad(out, [x, w], up)
    # a row's sums are made of some 32 terms a thread, then over threads: 16 u covers their roundings and the formula's
    for r in (0, 131072, 262144, n - 1):
        v = x.detach()[r].double()
        t = (v - v.mean()) / (v.var(correction=0) + 1e-5).sqrt()
        near = 2.0 ** -20 * (1 + t.abs()) * w.detach().double()
        assert ((out.detach()[r].double() - t * w.detach().double()).abs() <= near + 2.0 ** -8 * (t * w.detach()).abs()).all()
        g = up[r].double() * w.detach().double()
        want = (g - g.mean() - t * (g * t).mean()) / (v.var(correction=0) + 1e-5).sqrt()
        assert ((dx[r].double() - want).abs() <= 2.0 ** -20 * (1 + t.abs()) + 2.0 ** -8 * want.abs()).all()
    total = torch.zeros(d, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    for i in range(0, n, 4096):
        v = x.detach()[i:i + 4096].double()
        t = (v - v.mean(1, keepdim=True)) / (v.var(1, correction=0, keepdim=True) + 1e-5).sqrt()
        total += (up[i:i + 4096].double() * t).sum(0)
        size += (up[i:i + 4096].double() * t).abs().sum(0)
    assert ((dw.double() - total).abs() <= (ref.walk(n) + 2.0 ** -20) * size).all()


def test_large_embedding():
    import torch
    from paper_2608_24738_amd import training
    tokens, rows, width = 1200011, 400009, 4096
    announce("embedding %d of %d x %d bf16" % (tokens, rows, width))
    gen = torch.Generator(device="cuda").manual_seed(0)
    k = torch.randint(0, rows, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    k[-70000:] = rows - 1
    table = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda").uniform_(-1, 1, generator=gen).requires_grad_()
    out = training.embedding(k, table, scale=0.5)
    up = torch.empty_like(out).uniform_(-1, 1, generator=gen)
    grad, = torch.autograd.grad(out, table, up)
    for i in (0, 600000, 1048577, tokens - 1):
        assert torch.equal(out.detach()[i], (table.detach()[int(k[i])].float() * 0.5).bfloat16())
    for v in (0, 1, 200000, 262145, rows - 2, rows - 1):
        mine = up[k == v].double()
        ref.check(grad[v].double().cpu(), 0.5 * mine.sum(0).cpu(),
                  0.5 * ref.walk(len(mine)) * mine.abs().sum(0).cpu().numpy(), "row %d" % v, "bf16")
