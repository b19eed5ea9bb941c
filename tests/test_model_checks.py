"""The operators around a vocabulary refuse what they cannot do, on the host: no GPU is touched."""
import math

import pytest

from paper_2608_24738_amd import binding, training

(OK, NDIM, SHAPE, BATCH, NULL, NO_OUTPUT, SAMPLING, TOO_LARGE, ALIAS, UNSUPPORTED, HIP, METRIC, DTYPE,
 WORKSPACE) = range(0, -14, -1)
A, B, C, D, E, F, G, H = (0x10000000000 * (i + 1) for i in range(8))


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def head(lib, hidden=A, dtype=5, rows=40, classes=300, width=64, hs=64, weight=B, ws=64, labels=C, kind=3, scale=1.0,
         logp=D, sums=None, stats=None, room=E, nbytes=None):
    need = lib.tm_head_logp_workspace_size(dtype, rows, classes, width, weight, ws)
    return lib.tm_head_logp(hidden, dtype, rows, classes, width, hs, weight, ws, labels, kind, scale, logp, sums, stats,
                            room, need if nbytes is None else nbytes, None)


def test_head_checks(lib):
    for bad in (dict(rows=-1), dict(classes=0), dict(width=0), dict(hs=-64), dict(ws=-1)):
        assert head(lib, **bad) == SHAPE
    assert head(lib, dtype=3) == DTYPE and head(lib, kind=1) == DTYPE
    for scale in (0.0, -1.0, math.inf, math.nan, 1e39, 1e-39):
        assert head(lib, scale=scale) == SAMPLING
    for big in (dict(rows=1 << 31), dict(classes=1 << 31), dict(width=1 << 25), dict(rows=1 << 30, classes=1 << 30),
                dict(rows=1 << 26), dict(classes=1 << 30), dict(rows=1 << 25, classes=1 << 29),
                dict(classes=1 << 29, width=1 << 20, hs=1 << 20, ws=1 << 20),
                dict(hs=1 << 60), dict(ws=1 << 60)):
        assert head(lib, nbytes=1 << 50, **big) == TOO_LARGE
    assert head(lib, hidden=None) == NULL and head(lib, weight=None) == NULL
    assert head(lib, labels=None) == NULL
    assert head(lib, labels=None, logp=None) == NULL
    assert head(lib, logp=None) == NO_OUTPUT
    assert head(lib, room=None) == WORKSPACE and head(lib, room=E + 8) == WORKSPACE
    assert head(lib, nbytes=lib.tm_head_logp_workspace_size(5, 40, 300, 64, B, 64) - 1) == WORKSPACE
    for out in (dict(logp=A + 64), dict(logp=B + 64), dict(logp=C), dict(sums=D + 4), dict(stats=D - 4),
                dict(room=D), dict(room=A), dict(sums=A)):
        assert head(lib, **out) == ALIAS
    assert head(lib, rows=0) == OK and head(lib, rows=0, hidden=None, weight=None, room=None) == OK


def head_grad(lib, hidden=A, dtype=5, rows=40, classes=300, width=64, weight=B, labels=C, scale=1.0, stats=D, up=E,
              up_sum=None, dh=F, dw=G, room=H, nbytes=None):
    need = lib.tm_head_logp_grad_workspace_size(dtype, rows, classes, width, weight, width, dh is not None, dw is not None)
    return lib.tm_head_logp_grad(hidden, dtype, rows, classes, width, width, weight, width, labels, 3, scale, stats, up,
                                 up_sum, dh, dw, room, need if nbytes is None else nbytes, None)


def test_head_grad_checks(lib):
    assert head_grad(lib, dh=None, dw=None) == NO_OUTPUT
    assert head_grad(lib, up=None) == NULL and head_grad(lib, stats=None) == NULL and head_grad(lib, labels=None) == NULL
    assert head_grad(lib, hidden=None) == NULL
    assert head_grad(lib, scale=-2.0) == SAMPLING and head_grad(lib, dtype=0) == DTYPE
    assert head_grad(lib, width=0) == SHAPE
    assert head_grad(lib, room=None) == WORKSPACE and head_grad(lib, room=H + 4) == WORKSPACE
    assert head_grad(lib, nbytes=lib.tm_head_logp_grad_workspace_size(5, 40, 300, 64, B, 64, 1, 1) - 1) == WORKSPACE
    for out in (dict(dh=A), dict(dw=B + 2), dict(dh=E), dict(dw=F + 8), dict(room=F), dict(room=D), dict(dw=C), dict(dh=D)):
        assert head_grad(lib, **out) == ALIAS
    assert head_grad(lib, rows=0, dw=None) == OK


def test_head_workspaces(lib):
    """None for nothing, more where the weight has to be laid out, less for one gradient than for both."""
    size, grad = lib.tm_head_logp_workspace_size, lib.tm_head_logp_grad_workspace_size
    assert size(5, 0, 300, 64, A, 64) == 0 and grad(5, 0, 300, 64, A, 64, 1, 1) == 0
    assert size(9, 3, 300, 64, A, 64) == 0 and grad(9, 3, 300, 64, A, 64, 1, 1) == 0
    for rows in (1, 16, 17, 300, 5000, 100000):
        for dtype in (4, 5, 6):
            both = grad(dtype, rows, 50021, 777, A, 777, 1, 1)
            assert size(dtype, rows, 50021, 777, A, 777) > 0
            assert 0 < grad(dtype, rows, 50021, 777, A, 777, 1, 0) <= both
            assert 0 < grad(dtype, rows, 50021, 777, A, 777, 0, 1) <= both
    laid = 50176 * 1024 * 2
    for call in (lambda *w: size(5, 300, 50021, 1024, *w), lambda *w: grad(5, 300, 50021, 1024, *w, 1, 1)):
        assert call(A, 1024) + laid == call(A + 2, 1024) == call(A, 1025) == call(A, 1 << 23)
    # pieces of the vocabulary keep it far below a float32 for each logit
    assert grad(5, 8192, 131072, 2048, A, 2048, 1, 1) < 8192 * 131072 * 4 // 4


def norm(lib, x=A, dtype=5, rows=40, width=100, stride=100, weight=B, bias=C, params=6, eps=1e-5, out=D, stats=None):
    return lib.tm_layer_norm(x, dtype, rows, width, stride, weight, bias, params, eps, out, stats, None)


def test_norm_checks(lib):
    for bad in (dict(rows=-1), dict(width=0), dict(stride=-1)):
        assert norm(lib, **bad) == SHAPE
    assert norm(lib, dtype=3) == DTYPE and norm(lib, params=2) == DTYPE
    for eps in (0.0, -1e-5, math.inf, math.nan, 1e39, 1e-50):
        assert norm(lib, eps=eps) == SAMPLING
    for big in (dict(rows=1 << 31), dict(width=1 << 25), dict(stride=1 << 60)):
        assert norm(lib, **big) == TOO_LARGE
    assert norm(lib, x=None) == NULL and norm(lib, out=None) == NO_OUTPUT
    for out in (dict(out=A), dict(out=A + 7998), dict(out=B), dict(out=C + 396), dict(stats=D + 8), dict(stats=A)):
        assert norm(lib, **out) == ALIAS
    assert norm(lib, rows=0) == OK and norm(lib, rows=0, x=None, out=None) == OK


def norm_grad(lib, x=A, dtype=5, rows=40, width=100, weight=B, params=6, stats=C, up=D, dx=E, dw=F, db=G, room=H, nbytes=None):
    need = lib.tm_layer_norm_grad_workspace_size(dtype, rows, width)
    return lib.tm_layer_norm_grad(x, dtype, rows, width, width, weight, params, stats, up, dx, dw, db, room,
                                  need if nbytes is None else nbytes, None)


def test_norm_grad_checks(lib):
    assert norm_grad(lib, dx=None, dw=None, db=None) == NO_OUTPUT
    assert norm_grad(lib, stats=None) == NULL and norm_grad(lib, up=None) == NULL and norm_grad(lib, x=None) == NULL
    assert norm_grad(lib, params=1) == DTYPE and norm_grad(lib, width=0) == SHAPE
    assert norm_grad(lib, room=None) == WORKSPACE and norm_grad(lib, room=H + 4) == WORKSPACE
    assert norm_grad(lib, nbytes=lib.tm_layer_norm_grad_workspace_size(5, 40, 100) - 1) == WORKSPACE
    for out in (dict(dx=A), dict(dx=D), dict(dw=B), dict(db=F + 4), dict(dw=C), dict(room=E), dict(room=C), dict(dx=F - 4)):
        assert norm_grad(lib, **out) == ALIAS
    assert norm_grad(lib, rows=0, dw=None, db=None) == OK
    assert lib.tm_layer_norm_grad_workspace_size(5, 0, 100) == 0
    for rows, width in ((1, 1), (5, 100), (100000, 1000), (3, 40000)):
        assert lib.tm_layer_norm_grad_workspace_size(5, rows, width) >= 8 * width


def embed(lib, table=A, dtype=5, rows=40, width=100, stride=100, tokens=B, kind=3, count=9, scale=1.0, out=C):
    return lib.tm_embedding(table, dtype, rows, width, stride, tokens, kind, count, scale, out, None)


def test_embedding_checks(lib):
    for bad in (dict(rows=0), dict(width=0), dict(count=-1), dict(stride=-1)):
        assert embed(lib, **bad) == SHAPE
    assert embed(lib, dtype=2) == DTYPE and embed(lib, kind=6) == DTYPE
    for scale in (math.inf, math.nan, 1e39):
        assert embed(lib, scale=scale) == SAMPLING
    for big in (dict(rows=1 << 31), dict(rows=(1 << 31) - 1), dict(count=1 << 31), dict(width=1 << 25), dict(stride=1 << 60)):
        assert embed(lib, **big) == TOO_LARGE
    assert embed(lib, table=None) == NULL and embed(lib, tokens=None) == NULL and embed(lib, out=None) == NO_OUTPUT
    for out in (dict(out=A + 7998), dict(out=B + 71), dict(out=B - 1798)):
        assert embed(lib, **out) == ALIAS
    assert embed(lib, count=0) == OK and embed(lib, count=0, table=None, tokens=None, out=None) == OK


def embed_grad(lib, tokens=A, kind=3, count=9, up=B, dtype=5, rows=40, width=100, scale=1.0, out=C, room=D, nbytes=None):
    need = lib.tm_embedding_grad_workspace_size(rows, width, count)
    return lib.tm_embedding_grad(tokens, kind, count, up, dtype, rows, width, scale, out, room,
                                 need if nbytes is None else nbytes, None)


def test_embedding_grad_checks(lib):
    assert embed_grad(lib, out=None) == NO_OUTPUT
    assert embed_grad(lib, up=None) == NULL and embed_grad(lib, tokens=None) == NULL
    assert embed_grad(lib, dtype=0) == DTYPE and embed_grad(lib, scale=math.nan) == SAMPLING
    assert embed_grad(lib, room=None) == WORKSPACE and embed_grad(lib, room=D + 8) == WORKSPACE
    assert embed_grad(lib, nbytes=lib.tm_embedding_grad_workspace_size(40, 100, 9) - 1) == WORKSPACE
    for out in (dict(out=A + 71), dict(out=B + 1799), dict(room=C), dict(room=B)):
        assert embed_grad(lib, **out) == ALIAS
    assert lib.tm_embedding_grad_workspace_size(40, 100, 0) == 0
    for count in (1, 2048, 2049, 10 ** 6):
        assert lib.tm_embedding_grad_workspace_size(40, 100, count) >= 16 * count


def test_python_checks_without_a_gpu():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="ROCm"):
        training.head_log_probs(x, torch.zeros(9, 8), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="ROCm"):
        training.layer_norm(x)
    with pytest.raises(ValueError, match="ROCm"):
        training.embedding(torch.zeros(4, dtype=torch.int64), x)
