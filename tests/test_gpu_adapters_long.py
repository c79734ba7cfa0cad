"""First products of mwu_adapters_add that are longer than the 512 products after which a sum leaves the tensor core.

Tolerance, relative to a sum of positive products (whose running sum is half of it on average): 32 steps of a piece, each within 2^-22
of the running sum; the roundings of 2^-24 where the pieces are added, one after another (a CTA's pieces in four runs of warps in the
kernel for few rows) and over the CTAs; the second product, rank / 16 + 1 steps of 2^-22 a term; Y's own rounding."""
import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_gpu_adapters import Batch
from test_gpu_grouped import F64

pytestmark = pytest.mark.gpu


def worst(lengths, adapters, rank, rows, cols, ctas):
    """Largest relative error of Y over a batch of positive numbers, and its bound."""
    b = Batch(lengths, [s % adapters for s in range(len(lengths))], adapters, rank, rows, cols, 1, pad=False, with_scale=False)
    b.X[:, :cols].abs_()
    b.A[:, :rank, :cols].abs_()
    b.B[:, :rows, :rank].abs_()
    Y = torch.zeros_like(b.Y0)
    b.run(None, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    off = torch.zeros((), dtype=F64, device="cuda")
    for s in range(len(lengths)):
        rng, a = slice(b.at[s], b.at[s + 1]), b.which_list[s]
        t = torch.zeros(lengths[s], rank, dtype=F64, device="cuda")
        for k in range(0, cols, 1 << 17):
            t += b.X[rng, k:min(cols, k + (1 << 17))].to(F64) @ b.A[a, :rank, k:min(cols, k + (1 << 17))].to(F64).t()
        ref = t @ b.B[a, :rows, :rank].to(F64).t()
        off = torch.maximum(off, ((Y[rng, :rows].to(F64) - ref).abs() / ref).max())
    pieces = cols / ctas / 512 / 4 + 4
    bound = 16 * 2.0 ** -22 + (pieces + ctas) * 2.0 ** -25 + (rank / 16 + 1) * 3 * 2.0 ** -22 + 2.0 ** -24
    return float(off), bound


@pytest.mark.parametrize("rank,cols", [(3, 65536), (16, 65536), (24, 100000), (57, 40008), (128, 70003)])
@pytest.mark.parametrize("lengths", [[1], [3, 20, 9], [200], [33, 1, 260]], ids=str)
def test_long_sums(lengths, rank, cols):
    off, bound = worst(lengths, 2, rank, 40, cols, 1)
    assert off <= bound, (off, bound)


def test_as_many_columns_as_there_may_be():
    """Two CTAs to 16 rows: a warp's share of the columns is 65536, whose sum in one piece is 6e-5 off."""
    off, bound = worst([1] * 200, 200, 2, 8, B.MWU_MAX_GROUPED_SIDE, 2)
    # 16 * 2^-22 + 262 * 2^-25 + 3.4 * 2^-22 + 2^-24 = 1.25e-5, a fifth of that
    assert off <= bound < 6e-5 / 4, (off, bound)
