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
    need = lib.tm_head_logp_workspace_size(dtype, rows, classes, width)
    return lib.tm_head_logp(hidden, dtype, rows, classes, width, hs, weight, ws, labels, kind, scale, logp, sums, stats,
                            room, need if nbytes is None else nbytes, None)


def test_head_checks(lib):
    for bad in (dict(rows=-1), dict(classes=0), dict(width=0), dict(hs=-64), dict(ws=-1)):
        assert head(lib, **bad) == SHAPE
    assert head(lib, dtype=3) == DTYPE and head(lib, kind=1) == DTYPE
    for scale in (0.0, -1.0, math.inf, math.nan, 1e39, 1e-39):
        assert head(lib, scale=scale) == SAMPLING
    for big in (dict(rows=1 << 31), dict(classes=1 << 31), dict(width=1 << 25), dict(rows=1 << 30, classes=1 << 30),
                dict(hs=1 << 60), dict(ws=1 << 60)):
        assert head(lib, nbytes=1 << 50, **big) == TOO_LARGE
    assert head(lib, hidden=None) == NULL and head(lib, weight=None) == NULL
    assert head(lib, labels=None) == NULL
    assert head(lib, labels=None, logp=None) == NULL
    assert head(lib, logp=None) == NO_OUTPUT
    assert head(lib, room=None) == WORKSPACE and head(lib, room=E + 8) == WORKSPACE
    assert head(lib, nbytes=lib.tm_head_logp_workspace_size(5, 40, 300, 64) - 1) == WORKSPACE
    for out in (dict(logp=A + 64), dict(logp=B + 64), dict(logp=C), dict(sums=D + 4), dict(stats=D - 4),
                dict(room=D), dict(room=A), dict(sums=A)):
        assert head(lib, **out) == ALIAS
    assert head(lib, rows=0) == OK and head(lib, rows=0, hidden=None, weight=None, room=None) == OK


def head_grad(lib, hidden=A, dtype=5, rows=40, classes=300, width=64, weight=B, labels=C, scale=1.0, stats=D, up=E,
              up_sum=None, dh=F, dw=G, room=H, nbytes=None):
    need = lib.tm_head_logp_grad_workspace_size(dtype, rows, classes, width, dh is not None, dw is not None)
    return lib.tm_head_logp_grad(hidden, dtype, rows, classes, width, width, weight, width, labels, 3, scale, stats, up,
                                 up_sum, dh, dw, room, need if nbytes is None else nbytes, None)


def test_head_grad_checks(lib):
    assert head_grad(lib, dh=None, dw=None) == NO_OUTPUT
    assert head_grad(lib, up=None) == NULL and head_grad(lib, stats=None) == NULL and head_grad(lib, labels=None) == NULL
    assert head_grad(lib, hidden=None) == NULL
    assert head_grad(lib, scale=-2.0) == SAMPLING and head_grad(lib, dtype=0) == DTYPE
    assert head_grad(lib, width=0) == SHAPE
    assert head_grad(lib, room=None) == WORKSPACE and head_grad(lib, room=H + 4) == WORKSPACE
    assert head_grad(lib, nbytes=lib.tm_head_logp_grad_workspace_size(5, 40, 300, 64, 1, 1) - 1) == WORKSPACE
    for out in (dict(dh=A), dict(dw=B + 2), dict(dh=E), dict(dw=F + 8), dict(room=F), dict(room=D), dict(dw=C), dict(dh=D)):
        assert head_grad(lib, **out) == ALIAS
    assert head_grad(lib, rows=0, dw=None) == OK


def test_head_workspaces(lib):
    """One class more, one row more, another type: never less room, and none for nothing."""
    size, grad = lib.tm_head_logp_workspace_size, lib.tm_head_logp_grad_workspace_size
    assert size(5, 0, 300, 64) == 0 and grad(5, 0, 300, 64, 1, 1) == 0
    assert size(9, 3, 300, 64) == 0 and grad(9, 3, 300, 64, 1, 1) == 0
    for rows in (1, 16, 17, 300, 5000, 100000):
        for dtype in (4, 5, 6):
            both = grad(dtype, rows, 50021, 777, 1, 1)
            assert size(dtype, rows, 50021, 777) > 0
            assert 0 < grad(dtype, rows, 50021, 777, 1, 0) <= both and 0 < grad(dtype, rows, 50021, 777, 0, 1) <= both
    # pieces of the vocabulary keep it far below a float32 for each logit
    assert grad(5, 8192, 131072, 2048, 1, 1) < 8192 * 131072 * 4 // 4


def test_python_checks_without_a_gpu():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="ROCm"):
        training.head_log_probs(x, torch.zeros(9, 8), torch.zeros(4, dtype=torch.int64))
