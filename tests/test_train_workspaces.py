"""The workspaces that the training operators ask for, and their refusal of smaller ones: on the host, no GPU is touched."""
import ctypes

import pytest

from paper_2608_24738_amd import binding

WORKSPACE, ALIAS = -13, -8
A, B, C, D, E, F = (0x100000000 * (i + 1) for i in range(6))


def longs(*v):
    return (ctypes.c_int64 * len(v))(*v)


@pytest.mark.parametrize("dtype,classes,k", [(5, 200000, 4), (5, 32769, 1), (6, 131072, 32), (4, 50021, 0)])
def test_parts_of_a_row(dtype, classes, k):
    """A long row among few is cut into parts, which leave their sums (16 bytes) and k keys in the workspace."""
    lib = binding.load()
    need = lib.tm_label_logp_workspace_size(dtype, 1, classes, 1, longs(classes, 1, 1), k)
    assert need > 0 and need % (16 + 8 * k) == 0

    def call(ws, nbytes):
        return lib.tm_label_logp(A, dtype, 1, classes, 1, longs(classes, 1, 1), B, 3, None, None, k, C, None, None,
                                 D if k else None, E if k else None, None, ws, nbytes, None)
    assert call(None, need) == WORKSPACE
    assert call(F, need - 1) == WORKSPACE
    assert call(F + 4, need) == WORKSPACE
    assert call(A, need) == ALIAS
    assert call(C - 8, need) == ALIAS


def test_rows_without_parts():
    lib = binding.load()
    for outer, classes, inner in ((1, 32768, 1), (512, 50021, 1), (8, 4, 4096), (2, 150, 1000)):
        strides = longs(classes * inner, inner, 1)
        assert lib.tm_label_logp_workspace_size(5, outer, classes, inner, strides, 4) == 0


@pytest.mark.parametrize("buckets,heads", [(1, 1), (4, 3), (32, 16), (17, 17), (256, 65536)])
def test_partial_sums_of_a_table(buckets, heads):
    """Partial sums of 16 heads and all buckets, rounded up to 16 and a power of two, by at least 64 workgroups."""
    lib = binding.load()
    need = lib.tm_bias_grad_workspace_size(buckets, heads)
    rows = max(16, 1 << (buckets - 1).bit_length())
    groups = (heads + 15) // 16
    assert need >= 64 * groups * rows * 64 and need % (groups * rows * 64) == 0

    def field(ws, nbytes):
        return lib.tm_distance_bias_grad(A, 6, 2, 3, B, 6, buckets, heads, C, D, 6, ws, nbytes, None)

    def grid(ws, nbytes):
        return lib.tm_relative_bias_grad(1, longs(3), longs(4), None, 0, None, 1, B, 6, buckets, heads, C, D, 6, ws,
                                         nbytes, None)
    for call in (field, grid):
        assert call(None, need) == WORKSPACE
        assert call(1 << 50, need - 1) == WORKSPACE
        assert call((1 << 50) + 8, need) == WORKSPACE
        assert call(D - need + 16, need) == ALIAS
