"""Log-probabilities from hidden states and a vocabulary's weight, and their gradients, against float64."""
import numpy as np
import pytest

import head_reference as ref
from gpu_util import announce

pytestmark = pytest.mark.gpu

KINDS = {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}


def make(n, v, d, dtype, seed=0, pad=(0, 0), shift=(0, 0), kind="int64", missing=0.2):
    """Inputs whose rows are `pad` elements longer than the width and begin `shift` elements into their memory."""
    import torch
    gen = torch.Generator().manual_seed(1000 * seed + n + 7 * v + 13 * d)
    t = getattr(torch, KINDS[dtype])
    labels = torch.randint(0, v, (n,), generator=gen)
    weight = torch.randn(v, d, generator=gen) / max(1.0, d ** 0.5)
    hidden = torch.randn(n, d, generator=gen) + torch.rand(n, 1, generator=gen) * weight[labels] * d ** 0.5
    out = []
    for x, extra, first in ((hidden, pad[0], shift[0]), (weight, pad[1], shift[1])):
        flat = torch.full((first + x.shape[0] * (d + extra),), float("nan"), dtype=t, device="cuda")
        view = flat[first:].view(x.shape[0], d + extra)[:, :d]
        view.copy_(x.to(t))
        out.append(view)
    lost = torch.rand(n, generator=gen) < missing
    if kind == "uint8":
        labels = torch.where(lost | (labels > 255), torch.full_like(labels, 255), labels)
    else:
        labels = torch.where(lost, torch.tensor([-1, -100, v, v + 7])[torch.arange(n) % 4], labels)
    labels = labels.to(getattr(torch, kind)).cuda()
    ups = torch.randn(n, generator=gen), 0.1 * torch.randn(n, generator=gen)
    return out[0], out[1], labels, [u.cuda() for u in ups]


def run(hidden, weight, labels, ups, scale, log_sums):
    import torch
    from paper_2608_24738_amd import training
    h, w = hidden.detach().requires_grad_(), weight.detach().requires_grad_()
    got = training.head_log_probs(h, w, labels, scale=scale, log_sums=log_sums)
    outs = [got.log_probs] + ([got.log_sums] if log_sums else [])
    grads = torch.autograd.grad(outs, [h, w], ups[:len(outs)])
    torch.cuda.synchronize()
    return got, grads


def numbers(t):
    return t.detach().double().cpu().numpy()


def compare(hidden, weight, labels, ups, scale, log_sums, dtype, what):
    announce(what)
    got, (dh, dw) = run(hidden, weight, labels, ups, scale, log_sums)
    want = ref.exact(numbers(hidden), numbers(weight), labels.cpu().numpy(), scale, dtype,
                     (numbers(ups[0]), numbers(ups[1]) if log_sums else None), log_sums)
    ref.check(numbers(got.log_probs), want["logp"], want["tol_logp"], "log_probs")
    if log_sums:
        ref.check(numbers(got.log_sums), want["log_sum"], want["tol_log_sum"], "log_sums")
    else:
        assert got.log_sums is None
    ref.check(numbers(dh), want["dh"], want["tol_dh"], "hidden's gradient", dtype)
    ref.check(numbers(dw), want["dw"], want["tol_dw"], "weight's gradient", dtype)
    assert dh.dtype == hidden.dtype and dw.dtype == weight.dtype
    return got, dh, dw


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,d", [
    (1, 1, 1), (1, 1000, 64), (1, 4099, 257), (2, 17, 8), (4, 300, 1000), (5, 63, 16), (16, 1025, 129), (3, 70, 2049),
    (17, 1, 1), (17, 33, 7), (20, 130, 64), (64, 1000, 192), (127, 255, 72), (129, 257, 136), (300, 513, 96),
    (513, 777, 8), (260, 70, 300), (40, 5000, 31)])
def test_sizes(dtype, n, v, d):
    hidden, weight, labels, ups = make(n, v, d, dtype)
    compare(hidden, weight, labels, ups, 1.0, False, dtype, "head %s %dx%dx%d" % (dtype, n, v, d))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,d", [
    (6, 900, 264), (8, 777, 100), (9, 14, 2600), (300, 14, 2500), (600, 39, 1303), (90, 65, 1030), (1500, 20, 515),
    (20, 40000, 24), (33, 50001, 16), (4096, 9, 20), (4097, 9, 20), (2049, 3, 33)])
def test_waves_that_share_rows_and_many_splits(dtype, n, v, d):
    """Few classes of long rows, many classes of few and short ones, the numbers of rows where packing changes its way."""
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=2)
    compare(hidden, weight, labels, ups, 1.0, False, dtype, "head shared %s %dx%dx%d" % (dtype, n, v, d))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,d", [(1, 500, 96), (9, 100, 40), (33, 300, 64), (200, 700, 100)])
def test_log_sums_and_scale(dtype, n, v, d):
    hidden, weight, labels, ups = make(n, v, d, dtype, seed=1)
    compare(hidden, weight, labels, ups, 0.37, True, dtype, "head sums %s %dx%dx%d" % (dtype, n, v, d))


@pytest.mark.parametrize("n,v,d,pad,shift", [
    (2, 100, 64, (3, 5), (1, 1)), (2, 100, 64, (8, 8), (0, 8)), (50, 100, 64, (3, 0), (1, 0)), (50, 100, 64, (0, 5), (0, 0)),
    (50, 100, 64, (0, 8), (0, 1)), (50, 100, 61, (3, 3), (0, 0)), (200, 300, 200, (0, 56), (0, 8))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_alignment(dtype, n, v, d, pad, shift):
    """Rows that are parts of longer ones, beside which lies NaN, and that begin anywhere."""
    hidden, weight, labels, ups = make(n, v, d, dtype, pad=pad, shift=shift)
    compare(hidden, weight, labels, ups, 1.0, False, dtype, "head strides %s" % ((dtype, n, v, d, pad, shift),))


@pytest.mark.parametrize("kind", ["uint8", "int32", "int64"])
def test_label_types(kind):
    for n in (6, 70):
        hidden, weight, labels, ups = make(n, 255, 48, "bf16", kind=kind)
        compare(hidden, weight, labels, ups, 1.0, False, "bf16", "head labels %s %d" % (kind, n))


@pytest.mark.parametrize("n", [3, 8000])
def test_large_tiles_and_many_rows(n):
    """More rows than one workgroup packs, several parts of the products for dh, tiles of both sizes."""
    hidden, weight, labels, ups = make(n, 2100, 72, "bf16", missing=0.4)
    compare(hidden, weight, labels, ups, 1.0, False, "bf16", "head many %d" % n)
    hidden, weight, labels, ups = make(n, 2100, 72, "f16", missing=0.4)
    compare(hidden, weight, labels, ups, 1.0, False, "f16", "head many f16 %d" % n)


@pytest.mark.parametrize("d", [64, 60])
def test_pieces_of_the_vocabulary(d):
    """16384 rows of 16 bits: pieces of 4096 classes, the last one short; rows of 60 are laid out in whole steps."""
    hidden, weight, labels, ups = make(16300, 9000, d, "bf16", missing=0.97)
    compare(hidden, weight, labels, ups, 1.0, False, "bf16", "head pieces %d" % d)


@pytest.mark.parametrize("n", [5, 100])
def test_rows_without_labels_hold_anything(n):
    """NaN and infinities in rows without a label reach nothing."""
    import torch
    hidden, weight, labels, ups = make(n, 200, 40, "bf16", missing=0.4)
    lost = (labels < 0) | (labels >= 200)
    assert lost.any() and not lost.all()
    clean = run(hidden, weight, labels, ups, 1.0, False)
    dirty = hidden.clone()
    dirty[lost] = float("nan")
    dirty[lost.nonzero()[0]] = float("inf")
    ups = [torch.where(lost, torch.full_like(u, float("nan")), u) for u in ups]
    got = run(dirty, weight, labels, ups, 1.0, False)
    assert torch.equal(clean[0].log_probs, got[0].log_probs)
    for a, b in zip(clean[1], got[1]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n", [5, 100])
def test_no_labels_at_all(n):
    import torch
    hidden, weight, labels, ups = make(n, 200, 40, "f16", missing=2.0)
    got, (dh, dw) = run(hidden, weight, labels, ups, 1.0, False)
    assert not got.log_probs.any() and not dh.any() and not dw.any()
    got, (dh, dw) = run(hidden, weight, labels, ups, 1.0, True)
    assert not got.log_probs.any() and dh.isfinite().all() and dw.any()


@pytest.mark.parametrize("n", [5, 100])
def test_rows_that_are_not_finite(n):
    """NaN in a row makes that row NaN; a logit of -inf takes its class out of the sum."""
    import torch
    from paper_2608_24738_amd import training
    hidden, weight, labels, ups = make(n, 200, 40, "f32", missing=0.0)
    hidden = hidden.abs() + 0.5
    base = training.head_log_probs(hidden, weight, labels, log_sums=True)
    dirty = hidden.clone()
    dirty[2, 7] = float("nan")
    got = training.head_log_probs(dirty, weight, labels, log_sums=True)
    assert got.log_probs[2].isnan() and got.log_sums[2].isnan()
    keep = torch.arange(n, device="cuda") != 2
    assert torch.equal(got.log_probs[keep], base.log_probs[keep])
    heavy = weight.clone()
    heavy[150:] = -float("inf")
    y = labels % 150
    got = training.head_log_probs(hidden, heavy, y, log_sums=True)
    short = training.head_log_probs(hidden, weight[:150].contiguous(), y, log_sums=True)
    assert torch.allclose(got.log_probs, short.log_probs, rtol=0, atol=1e-5)
    heavy[:] = -float("inf")
    got = training.head_log_probs(hidden, heavy, y, log_sums=True)
    assert (got.log_probs == -float("inf")).all() and (got.log_sums == -float("inf")).all()


def test_far_logits():
    """Logits of some +-1000: nothing overflows, and p near 1 keeps its gradient's sign and zeros."""
    for n in (4, 60):
        hidden, weight, labels, ups = make(n, 300, 64, "bf16", missing=0.0)
        compare(hidden * 100, weight * 4, labels, ups, 1.0, True, "bf16", "head far %d" % n)


@pytest.mark.parametrize("n", [3, 90])
def test_wide_range_of_upstream_gradients(n):
    """Upstream gradients over 2^20 of range: float16 holds each row's as a multiple of its own power of two."""
    import torch
    hidden, weight, labels, ups = make(n, 300, 64, "f16", missing=0.1)
    sizes = torch.logspace(-3, 3, n, device="cuda")
    compare(hidden, weight, labels, [ups[0] * sizes, ups[1] * sizes], 1.0, True, "f16", "head range %d" % n)


@pytest.mark.parametrize("n", [2, 50])
def test_one_gradient_alone(n):
    import torch
    from paper_2608_24738_amd import training
    hidden, weight, labels, ups = make(n, 150, 40, "bf16")
    _, (dh, dw) = run(hidden, weight, labels, ups, 1.0, False)
    for which in (0, 1):
        leaves = [hidden.detach().clone(), weight.detach().clone()]
        leaves[which].requires_grad_()
        got = training.head_log_probs(*leaves, labels)
        grad, = torch.autograd.grad(got.log_probs, leaves[which], ups[0])
        assert torch.equal(grad, (dh, dw)[which])


@pytest.mark.parametrize("n", [3, 70])
def test_shapes_and_broadcast_rows(n):
    """Leading axes, no rows at all, one row repeated by a stride of zero, a transposed weight."""
    import torch
    from paper_2608_24738_amd import training
    hidden, weight, labels, ups = make(2 * n, 150, 40, "bf16")
    flat = training.head_log_probs(hidden, weight, labels)
    many = training.head_log_probs(hidden.view(2, n, 40), weight, labels.view(2, n))
    assert torch.equal(many.log_probs.view(-1), flat.log_probs)
    turned = weight.t().contiguous().t()
    assert torch.equal(training.head_log_probs(hidden, turned, labels).log_probs, flat.log_probs)
    swapped = hidden.view(2, n, 40).transpose(0, 1)
    assert torch.equal(training.head_log_probs(swapped, weight, labels.view(2, n).t()).log_probs.t().reshape(-1), flat.log_probs)
    row = hidden[:1].detach().requires_grad_()
    got = training.head_log_probs(row.expand(2 * n, 40), weight, labels)
    got.log_probs.sum().backward()
    one = training.head_log_probs(row.detach().repeat(2 * n, 1), weight, labels)
    assert torch.equal(got.log_probs, one.log_probs) and row.grad.shape == row.shape
    w = weight.detach().requires_grad_()
    none = training.head_log_probs(hidden[:0], w, labels[:0])
    assert none.log_probs.shape == (0,)
    none.log_probs.sum().backward()
    assert not w.grad.any()


def test_difference_quotients():
    """The gradients against differences of the log-probabilities in float64's plain form, along random directions."""
    import torch
    for n in (5, 40):
        hidden, weight, labels, ups = make(n, 90, 24, "f32", missing=0.2)
        _, (dh, dw) = run(hidden, weight, labels, ups, 0.7, True)
        gen = torch.Generator().manual_seed(5)
        h, w = hidden.double().cpu(), weight.double().cpu()
        y = labels.cpu()
        has = (y >= 0) & (y < 90)

        def value(h, w):
            x = float(np.float32(0.7)) * (h @ w.t())
            total = torch.logsumexp(x, 1)
            l = torch.where(has, x.gather(1, torch.where(has, y, 0)[:, None])[:, 0] - total, 0.0)
            return (ups[0].double().cpu() * l + ups[1].double().cpu() * total).sum()
        for _ in range(4):
            eh, ew = torch.randn(h.shape, generator=gen).double(), torch.randn(w.shape, generator=gen).double()
            step = 1e-5
            slope = (value(h + step * eh, w + step * ew) - value(h - step * eh, w - step * ew)) / (2 * step)
            have = (dh.double().cpu() * eh).sum() + (dw.double().cpu() * ew).sum()
            size = (dh.double().cpu() * eh).abs().sum() + (dw.double().cpu() * ew).abs().sum()
            # float32 gradients are off by some 100 u of their sizes, the quotient by 1e-10 of third derivatives
            assert abs(slope - have) <= 2.0 ** -17 * size + 1e-7


def test_two_calls_give_the_same_bits():
    import torch
    for n in (7, 900):
        hidden, weight, labels, ups = make(n, 3000, 136, "bf16")
        a, b = (run(hidden, weight, labels, ups, 1.0, True) for _ in range(2))
        for x, y in zip(list(a[0]) + list(a[1]), list(b[0]) + list(b[1])):
            assert torch.equal(x, y)


@pytest.mark.parametrize("n", [4, 80])
def test_captured_and_replayed(n):
    """A forward and backward pass in a graph, replayed on new values between eager calls."""
    import torch
    from paper_2608_24738_amd import training
    hidden, weight, labels, ups = make(n, 700, 72, "bf16")
    h, w = hidden.detach().clone().requires_grad_(), weight.detach().clone().requires_grad_()

    def step():
        got = training.head_log_probs(h, w, labels)
        return (got.log_probs,) + torch.autograd.grad(got.log_probs, [h, w], ups[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        new = make(n, 700, 72, "bf16", seed=10 + i)
        with torch.no_grad():
            h.copy_(new[0])
            w.copy_(new[1])
            labels.copy_(new[2])
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.detach().clone() for t in out]
        for a, b in zip(kept, run(h, w, labels, ups, 1.0, False)[1]):
            pass
        eager = run(h, w, labels, ups, 1.0, False)
        for a, b in zip(kept, [eager[0].log_probs] + list(eager[1])):
            assert torch.equal(a, b)


def test_another_stream():
    import torch
    hidden, weight, labels, ups = make(300, 900, 64, "bf16")
    want = run(hidden, weight, labels, ups, 1.0, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(hidden, weight, labels, ups, 1.0, False)
    side.synchronize()
    assert torch.equal(want[0].log_probs, got[0].log_probs)
    for a, b in zip(want[1], got[1]):
        assert torch.equal(a, b)
