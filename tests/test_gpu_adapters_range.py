"""mwu_adapters_add at the ends of the range of numbers: infinities of X A^T, and numbers of it that bf16 cannot hold."""
import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_gpu_adapters import Batch
from test_gpu_grouped import F64

pytestmark = pytest.mark.gpu

LENGTHS = [[3], [20, 1], [300], [1, 150, 2, 40]]        # the kernel for few rows, the one for many, both
RANKS = [1, 5, 16, 24, 57, 100, 128]


def one_sign(b):
    """A positive; the rows of B positive and negative in turn: a positive infinity of X gives infinities in Y, by the formula too."""
    b.A[:, :b.r, :b.k] = b.A[:, :b.r, :b.k].abs() + 2.0 ** -9
    sign = torch.ones(b.n, 1, device="cuda", dtype=torch.bfloat16)
    sign[1::2] = -1
    b.B[:, :b.n, :b.r] = (b.B[:, :b.n, :b.r].abs() + 2.0 ** -9) * sign


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_infinities_of_x(lengths, rank, fp32):
    rows, cols = 72, 136
    b = Batch(lengths, [s % 2 for s in range(len(lengths))], 2, rank, rows, cols, fp32, with_scale=False)
    one_sign(b)
    sick = sorted({0, b.M // 2, b.M - 1})
    for i, m in enumerate(sick):
        b.X[m, (37 * i) % cols] = float("inf") if i % 2 == 0 else -float("inf")
    for Y0 in (None, b.Y0):
        Y = torch.zeros_like(b.Y0)
        b.run(Y0, Y)
        torch.cuda.synchronize()
        assert int(b.st.item()) == 0
        for i, m in enumerate(sick):
            want = torch.full((rows,), float("inf") if i % 2 == 0 else -float("inf"), device="cuda")
            want[1::2] *= -1
            assert torch.equal(Y[m, :rows].float(), want), (m, Y[m, :8])
        well = [m for m in range(b.M) if m not in sick]
        assert bool(torch.isfinite(Y[well, :rows]).all())


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_numbers_that_round_to_an_infinity(lengths, rank, fp32):
    """X A^T = +-(2 - 2^-9) 2^127: an fp32 number whose nearest bf16 is an infinity; B of 2^-100 brings Y back into range.

    T is exact, its first two terms hold it exactly, and so is a sum of equal T b over the rank up to the tensor core's 2^-22 a step
    of the running magnitude; a bf16 Y rounds by 2^-8."""
    rows, cols = 40, 72
    b = Batch(lengths, [0] * len(lengths), 1, rank, rows, cols, fp32, with_scale=False)
    b.X[:, :cols] = 0
    b.A[:, :rank, :cols] = 0
    b.X[:b.M, 1], b.X[:b.M, 40] = 2.0 ** 64, 2.0 ** 64
    b.A[:, :rank, 1], b.A[:, :rank, 40] = (2 - 2.0 ** -7) * 2.0 ** 63, (2.0 ** -8 + 2.0 ** -9) * 2.0 ** 63
    b.X[1::2] *= -1
    b.B[:, :rows, :rank] = 2.0 ** -100
    Y = torch.zeros_like(b.Y0)
    b.run(None, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    ref = torch.full((b.M, rows), (2 - 2.0 ** -9) * 2.0 ** 27 * rank, dtype=F64, device="cuda")
    ref[1::2] *= -1
    steps = (rank / 16 + 1) * (3 if fp32 else 2)
    tol = ref.abs() * (steps * 2.0 ** -22 + 2.0 ** -23 + (0 if fp32 else 2.0 ** -8))
    assert bool(((Y[:, :rows].to(F64) - ref).abs() <= tol).all())
