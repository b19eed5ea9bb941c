"""Log-probabilities from hidden states where the vocabulary is taken in pieces, and bounds of few rows, against float64."""
import pytest

import head_reference as ref
from gpu_util import announce
from test_gpu_head import compare, make, numbers, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,v,d,dtype,sums", [(8200, 9000, 40, "f16", True), (8200, 9000, 61, "f16", False),
                                              (4200, 12000, 40, "f32", False), (4200, 12000, 33, "f32", True)])
def test_gradient_in_pieces(n, v, d, dtype, sums):
    """g of up to 128 MB a piece: two pieces of 4608 classes for 8448 rows of float16, three of 4096 for 4352 rows of planes."""
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=12, missing=0.3)
    compare(hidden, weight, labels, ups, 1.0, sums, dtype, "head pieces %s %dx%dx%d" % (dtype, n, v, d))


@pytest.mark.parametrize("n,v,d,dtype", [(40, 600011, 1001, "bf16"), (300, 600011, 1001, "f16"), (140, 200011, 1000, "f32")])
def test_weights_laid_out_in_pieces(n, v, d, dtype):
    """Rows that tiles cannot read in place, more of them than 1 GiB holds: two pieces, with labels and mass in both."""
    import torch
    from paper_2608_24738_amd import training
    announce("head laid pieces %s %dx%dx%d" % (dtype, n, v, d))
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = torch.empty((v, d), dtype=t, device="cuda").uniform_(-0.05, 0.05, generator=gen)
    y = torch.randint(0, 500, (n,), generator=gen, device="cuda")
    y[1::2] = v - 1 - y[1::2]
    h = torch.randn((n, d), generator=gen, device="cuda")
    # a row's mass: half at its label, as much in the other piece
    h = (h + 14 * w[y].float() + 14 * w[(v - 1 - y) % v].float()).to(t)
    y[5] = -1
    up = torch.randn(n, generator=gen, device="cuda")
    leaves = [h.requires_grad_(), w.requires_grad_()]
    got = training.head_log_probs(*leaves, y, log_sums=True)
    dh, dw = torch.autograd.grad(got.log_probs, leaves, up)
    with torch.no_grad():
        hd, step = h.double(), 50000
        x = torch.cat([hd @ w[i:i + step].double().t().contiguous() for i in range(0, v, step)], 1)
        size = torch.stack([(hd.abs() @ w[i:i + step].double().abs().t().contiguous()).max() for i in range(0, v, step)]).max()
        total = torch.logsumexp(x, 1)
        has = y >= 0
        want = torch.where(has, x.gather(1, y.clamp_min(0)[:, None])[:, 0] - total, 0.0)
        off = 2 * ref.walk(d) * float(size) + 2 * ref.U * float(x.abs().max()) + ref.walk(v, 8)
        assert (got.log_sums.double() - total).abs().max() <= off + 4 * ref.U * float(total.abs().max())
        assert (got.log_probs.double() - want).abs().max() <= off + 4 * ref.U * float(want.abs().max())
        a = torch.where(has, up.double(), 0.0)
        g = -a[:, None] * (x - total[:, None]).exp()
        g[torch.arange(n), y.clamp_min(0)] += a
        # slopes are off by `off` relatively, and by half a step of the type, or of two numbers of it
        half = ref.HALF[dtype] if n > 256 else ref.HALF[dtype] ** 2
        tol = (8 * ref.U + half) * g.abs()
        tol += 2.0 ** -126 * (1 + a.abs())[:, None]
        if dtype == "f16":
            tol += 2.0 ** -25 * 2.0 ** -14 * 2 * float(a.abs().max())
        tol += off * (g.abs() + a.abs()[:, None] * (x - total[:, None]).exp())
        for rows in (slice(0, 500), slice(299000, 301000), slice(v - 500, v)):
            rows = slice(min(rows.start, v - 500), rows.stop)
            ref.check(numbers(dw[rows]), numbers(g[:, rows].t().contiguous() @ hd),
                      numbers(tol[:, rows].t().contiguous() @ hd.abs() + ref.walk(n) * (g[:, rows].abs().t().contiguous() @ hd.abs())),
                      "weight's gradient", dtype)
        exact, room = torch.zeros((n, d), dtype=torch.float64, device="cuda"), 0.0
        for i in range(0, v, step):
            part = w[i:i + step].double()
            exact += g[:, i:i + step] @ part
            room = room + (tol[:, i:i + step] + ref.walk(v) * g[:, i:i + step].abs()) @ part.abs()
        ref.check(numbers(dh), numbers(exact), numbers(room), "hidden's gradient", dtype)
        assert not dh[5].any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [5, 6, 7, 8])
def test_few_rows_keep_g_in_float32(dtype, n):
    """Up to eight rows of 16 bits, whose slopes are not rounded: the bounds of float32 operands, results rounded once."""
    hidden, weight, labels, ups = make(n, 900, 136, dtype, seed=13)
    announce("few rows %s %d" % (dtype, n))
    _, (dh, dw) = run(hidden, weight, labels, ups, 0.8, True)
    want = ref.exact(numbers(hidden), numbers(weight), labels.cpu().numpy(), 0.8, "f32", (numbers(ups[0]), numbers(ups[1])), True)
    ref.check(numbers(dh), want["dh"], want["tol_dh"], "hidden's gradient", dtype)
    ref.check(numbers(dw), want["dw"], want["tol_dw"], "weight's gradient", dtype)


def test_two_calls_at_once():
    """Two streams with their own workspaces, and rows of both kinds, give what each gives alone."""
    import torch
    cases = [make(300, 3000, 136, "bf16", seed=14), make(6, 3000, 136, "bf16", seed=15), make(200, 3000, 61, "f32", seed=16)]
    alone = [run(*case, 1.0, False) for case in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    from paper_2608_24738_amd import training
    got = []
    for _ in range(5):
        for i, (case, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                h, w = case[0].detach().requires_grad_(), case[1].detach().requires_grad_()
                out = training.head_log_probs(h, w, case[2])
                got.append((i, out.log_probs, torch.autograd.grad(out.log_probs, [h, w], case[3][0])))
    torch.cuda.synchronize()
    for i, logp, grads in got:
        assert torch.equal(logp, alone[i][0].log_probs)
        assert all(torch.equal(a, b) for a, b in zip(grads, alone[i][1]))
