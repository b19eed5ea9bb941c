"""What the gradient's workspace holds: a copy of the weight where something reads it, on the host."""
import pytest

from paper_2608_24738_amd import binding

A = 0x10000000000


@pytest.mark.parametrize("dtype,size", [(4, 2), (5, 2)])
@pytest.mark.parametrize("rows,classes,width", [(20, 300, 128), (300, 513, 512), (64, 1500, 4032), (1000, 60, 256)])
def test_weights_that_nothing_reads_take_no_room(dtype, size, rows, classes, width):
    """Rows of whole 128 bytes, aligned and not: the copy is for dh; the weight's gradient by single waves needs none."""
    grad = binding.load().tm_head_logp_grad_workspace_size
    laid = -(-classes // 256) * 256 * width * size
    for hidden, weight in ((1, 0), (1, 1)):
        assert grad(dtype, rows, classes, width, A + 2, width, hidden, weight) == laid + grad(
            dtype, rows, classes, width, A, width, hidden, weight)
    assert grad(dtype, rows, classes, width, A + 2, width, 0, 1) == grad(dtype, rows, classes, width, A, width, 0, 1)


def test_weights_that_tiles_read():
    """Large problems take the logits by tiles, which read the copy."""
    grad = binding.load().tm_head_logp_grad_workspace_size
    laid = 50176 * 1024 * 2
    assert grad(5, 300, 50021, 1024, A + 2, 1024, 0, 1) == laid + grad(5, 300, 50021, 1024, A, 1024, 0, 1)
