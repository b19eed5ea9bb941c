"""The training operators refuse what they cannot do, on the host: no GPU is touched."""
import ctypes

import pytest

from paper_2608_24738_amd import binding, training

(OK, NDIM, SHAPE, BATCH, NULL, NO_OUTPUT, SAMPLING, TOO_LARGE, ALIAS, UNSUPPORTED, HIP, METRIC, DTYPE,
 WORKSPACE) = range(0, -14, -1)
A, B, C, D, E, F = (0x100000000 * (i + 1) for i in range(6))


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def longs(*v):
    return (ctypes.c_int64 * len(v))(*v)


def logp(lib, shape=(2, 5, 7), dtype=6, strides=(35, 7, 1), labels=B, label_dtype=3, field=None, field_strides=None,
         k=0, logits=A, out=C, entropy=None, mean=None, top=None, index=None, stats=None, ws=None, ws_bytes=0):
    return lib.tm_label_logp(logits, dtype, *shape, longs(*strides) if strides else None, labels, label_dtype, field,
                             longs(*field_strides) if field_strides else None, k, out, entropy, mean, top, index,
                             stats, ws, ws_bytes, None)


def test_label_checks(lib):
    assert logp(lib, shape=(2, 0, 7)) == SHAPE
    assert logp(lib, shape=(-1, 5, 7)) == SHAPE
    assert logp(lib, strides=None) == SHAPE
    assert logp(lib, strides=(35, -7, 1)) == SHAPE
    assert logp(lib, field=D) == SHAPE                             # a field without strides
    assert logp(lib, dtype=7) == DTYPE
    assert logp(lib, label_dtype=1) == DTYPE
    assert logp(lib, shape=(1 << 16, 5, 1 << 16)) == TOO_LARGE
    assert logp(lib, strides=(1 << 62, 7, 1)) == TOO_LARGE
    assert logp(lib, logits=None) == NULL
    assert logp(lib, labels=None) == NULL
    assert logp(lib, mean=D) == NULL
    assert logp(lib, out=None) == NO_OUTPUT
    assert logp(lib, k=2) == NO_OUTPUT
    assert logp(lib, k=6, top=D, index=E) == UNSUPPORTED
    assert logp(lib, shape=(1, 50, 1), strides=(50, 1, 1), k=33, top=D, index=E) == UNSUPPORTED
    assert logp(lib, k=-1) == UNSUPPORTED
    assert logp(lib, out=A + 64) == ALIAS
    assert logp(lib, entropy=C + 4) == ALIAS
    assert logp(lib, out=B) == ALIAS
    assert logp(lib, shape=(0, 5, 7)) == OK and logp(lib, shape=(3, 5, 0), logits=None) == OK
    need = lib.tm_label_logp_workspace_size(5, 1, 200000, 1, longs(200000, 1, 1), 4)
    if need:
        assert logp(lib, shape=(1, 200000, 1), dtype=5, strides=(200000, 1, 1), k=4, top=D, index=E) == WORKSPACE
        assert logp(lib, shape=(1, 200000, 1), dtype=5, strides=(200000, 1, 1), k=4, top=D, index=E, ws=F + 4,
                    ws_bytes=need) == WORKSPACE
        assert logp(lib, shape=(1, 200000, 1), dtype=5, strides=(200000, 1, 1), k=4, top=D, index=E, ws=A,
                    ws_bytes=need) == ALIAS


def grad(lib, shape=(2, 5, 7), dtype=6, strides=(35, 7, 1), labels=B, field=None, field_strides=None, stats=None,
         entropy=None, mean=None, ua=D, uh=None, uf=None, out=E, out_strides=(35, 7, 1)):
    return lib.tm_label_logp_grad(A, dtype, *shape, longs(*strides), labels, 3, field,
                                  longs(*field_strides) if field_strides else None, stats, entropy, mean, ua, uh, uf,
                                  out, longs(*out_strides) if out_strides else None, None)


def test_label_grad_checks(lib):
    assert grad(lib, out_strides=None) == SHAPE
    assert grad(lib, out_strides=(35, -7, 1)) == SHAPE
    assert grad(lib, out_strides=(35, 0, 1)) == ALIAS              # classes on top of each other
    assert grad(lib, out_strides=(6, 7, 1)) == ALIAS
    assert grad(lib, ua=None) == NULL
    assert grad(lib, labels=None) == NULL
    assert grad(lib, uf=F) == NULL                                 # no field
    assert grad(lib, shape=(2, 33, 7), strides=(231, 7, 1), out_strides=(231, 7, 1)) == NULL   # no statistics
    assert grad(lib, stats=C, uh=F) == NULL                        # statistics without the entropy
    assert grad(lib, out=None) == NO_OUTPUT
    assert grad(lib, out=A) == ALIAS
    assert grad(lib, out=D) == ALIAS
    assert grad(lib, dtype=3) == DTYPE
    assert grad(lib, shape=(0, 5, 7)) == OK


def field_bias(lib, distances=A, kind=6, batch=2, positions=10, table=B, table_dtype=6, buckets=4, heads=3, edges=C,
               add=None, out=D, dtype=6):
    return lib.tm_distance_bias(distances, kind, batch, positions, table, table_dtype, buckets, heads, edges, add, out,
                                dtype, None)


def grid_bias(lib, query=(3, 4), key=(3, 4), offset=None, metric=0, sampling=None, batch=1, heads=3, add=None, out=D,
              ndim=None, buckets=4):
    samp = (ctypes.c_double * len(sampling))(*sampling) if sampling else None
    return lib.tm_relative_bias(len(query) if ndim is None else ndim, longs(*query) if query else None,
                                longs(*key) if key else None, longs(*offset) if offset else None, metric, samp, batch,
                                B, 6, buckets, heads, C, add, out, 6, None)


def test_bias_checks(lib):
    assert field_bias(lib, kind=3) == DTYPE
    assert field_bias(lib, table_dtype=7) == DTYPE
    assert field_bias(lib, dtype=2) == DTYPE
    assert field_bias(lib, buckets=0) == SHAPE
    assert field_bias(lib, buckets=257) == SHAPE
    assert field_bias(lib, heads=0) == SHAPE
    assert field_bias(lib, batch=-1) == SHAPE
    assert field_bias(lib, positions=1 << 31) == TOO_LARGE
    assert field_bias(lib, heads=1 << 30) == TOO_LARGE
    assert field_bias(lib, distances=None) == NULL
    assert field_bias(lib, edges=None) == NULL
    assert field_bias(lib, table=None) == NULL
    assert field_bias(lib, out=None) == NO_OUTPUT
    assert field_bias(lib, out=A + 8) == ALIAS
    assert field_bias(lib, add=D + 8) == ALIAS
    assert field_bias(lib, positions=0) == OK
    assert grid_bias(lib, ndim=0) == NDIM and grid_bias(lib, ndim=9) == NDIM
    assert grid_bias(lib, query=(), ndim=1) == SHAPE
    assert grid_bias(lib, query=(3, -4)) == SHAPE
    assert grid_bias(lib, batch=2) == SHAPE                        # a batch without scores
    assert grid_bias(lib, metric=4) == METRIC
    assert grid_bias(lib, metric=3) == METRIC                      # signed offsets have one axis
    assert grid_bias(lib, sampling=(1.0, 0.0)) == SAMPLING
    assert grid_bias(lib, sampling=(1.0, float("nan"))) == SAMPLING
    assert grid_bias(lib, sampling=(1.0, 1e300)) == SAMPLING
    assert grid_bias(lib, query=(5,), key=(5,), metric=3, sampling=(2.0,)) == SAMPLING
    assert grid_bias(lib, offset=(0, 1 << 31)) == TOO_LARGE
    assert grid_bias(lib, query=(1 << 20, 1 << 12)) == TOO_LARGE
    assert grid_bias(lib, out=C) == ALIAS
    assert grid_bias(lib, query=(0, 4)) == OK


def test_bias_grad_checks(lib):
    def call(buckets=4, heads=3, grad=B, out=D, ws=E, ws_bytes=1 << 40, batch=2, positions=10, dtype=6):
        return lib.tm_distance_bias_grad(A, 6, batch, positions, grad, dtype, buckets, heads, C, out, 6, ws, ws_bytes,
                                         None)
    assert call(buckets=300) == SHAPE
    assert call(dtype=0) == DTYPE
    assert call(grad=None) == NULL
    assert call(out=None) == NO_OUTPUT
    assert call(out=B) == ALIAS
    if lib.tm_bias_grad_workspace_size(4, 3):
        assert call(ws=None) == WORKSPACE
        assert call(ws=E + 8) == WORKSPACE
        assert call(ws_bytes=4) == WORKSPACE
        assert call(ws=D) == ALIAS


def test_wrappers_refuse():
    import torch
    x = torch.zeros((2, 5, 7))
    y = torch.zeros((2, 7), dtype=torch.int64)
    with pytest.raises(ValueError):
        training.label_log_probs(x, y)                             # not on the GPU
    table = torch.zeros((4, 2))
    with pytest.raises(ValueError):
        training.relative_bias(table, torch.zeros(3), 4, 4)
    with pytest.raises(ValueError):
        training.distance_bias(torch.zeros((1, 4)), table, torch.zeros(3))
    with pytest.raises(ValueError):
        training.distance_edges(0, 4.0)
    with pytest.raises(ValueError):
        training.distance_edges(257, 4.0)


@pytest.mark.parametrize("signed", [False, True])
@pytest.mark.parametrize("buckets", [1, 2, 3, 4, 7, 16, 31, 32, 255, 256])
def test_edges(buckets, signed):
    edges = training.distance_edges(buckets, 100.0, signed=signed).tolist()
    assert len(edges) == buckets - 1
    assert all(a < b for a, b in zip(edges, edges[1:]))


def test_collapse():
    assert training._collapse((2, 3, 4), (12, 4, 1)) == (24, 1)
    assert training._collapse((2, 3, 4), (24, 4, 1)) is None
    assert training._collapse((2, 1, 4), (4, 99, 1)) == (8, 1)
    assert training._collapse((), ()) == (1, 0)
    assert training._collapse((5, 1), (7, 3)) == (5, 7)
    assert training._collapse((3, 4), (0, 0)) == (12, 0)
    assert training._collapse((3, 4), (0, 1)) is None


def test_constants_match_the_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "tm_train.h"), encoding="utf-8") as f:
        text = f.read()
    value = {name: int(number) for name, number in re.findall(r"(TM_[A-Z_]+) = (\d+)", text)}
    assert training.MAX_TOP == value["TM_LABEL_MAX_TOP"]
    assert training.MAX_RECOMPUTE == value["TM_LABEL_MAX_RECOMPUTE"]
    assert training.MAX_BUCKETS == value["TM_BIAS_MAX_BUCKETS"]
    assert training.BIAS_METRICS["offset"] == value["TM_METRIC_OFFSET"]
