"""mwu_adapters_add where many boxes of a tile are not whole: rows that end inside 32, columns that end inside a chunk, several items to a
cluster, so that slots of the ring go round while such boxes leave."""
import pytest
import torch

from test_gpu_adapters import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("rank,rows,cols", [(16, 201, 520), (64, 1003, 200), (100, 333, 72), (128, 77, 1000)])
def test_boxes_that_are_not_whole(rank, rows, cols, fp32):
    lengths = [33 + (7 * s) % 100 for s in range(400)]
    b = Batch(lengths, [s % 6 - 1 for s in range(400)], 5, rank, rows, cols, fp32, pad=rows % 2 == 0)
    Z = b.Y0.clone()
    b.run(Z, Z)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    b.check(Z, b.Y0, b.Y0)
    want = Z
    for _ in range(20):
        Z = b.Y0.clone()
        b.run(Z, Z)
        assert torch.equal(Z, want)
