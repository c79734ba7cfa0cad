"""Grouped products and adapters on views of wider buffers, as a model holds them: several projections' inputs or outputs side by side."""
import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_gpu_adapters import Batch
from test_gpu_grouped import F64, check, gen_of, new_status, normal, offsets_of

pytestmark = pytest.mark.gpu


def test_grouped_products_on_views():
    lengths, rows, cols = [40, 0, 130, 7], 72, 136
    gen, at = gen_of(21), offsets_of(lengths)
    m, off, st, g = at[-1], torch.tensor(at, dtype=torch.int32, device="cuda"), new_status(), len(lengths)
    XX, DD, WW = normal(gen, m, 3 * cols), normal(gen, m, 2 * rows), normal(gen, g, 2, rows, cols, std=0.1)
    YY, GG = torch.full((m, 2 * rows), 7.0, device="cuda"), torch.full((g, 2, rows, cols), 7.0, device="cuda")
    X, dY, W, Y, dW = XX[:, cols:2 * cols], DD[:, rows:], WW[:, 1], YY[:, :rows], GG[:, 1]
    B.mwu_gemm_grouped(g, rows, cols, W, cols, 2 * rows * cols, off, X, m, 3 * cols, Y, 2 * rows, 1, st)
    B.mwu_gemm_grouped_dw(g, rows, cols, off, dY, m, 2 * rows, X, 3 * cols, dW, cols, 2 * rows * cols, 1, 0, st)
    dX = torch.full((m, 2 * cols), 7.0, device="cuda")
    B.mwu_gemm_grouped_dx(g, rows, cols, W, cols, 2 * rows * cols, off, dY, m, 2 * rows, dX[:, cols:], 2 * cols, 1, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert bool((YY[:, rows:] == 7).all() & (GG[:, 0] == 7).all() & (dX[:, :cols] == 7).all())
    for i in range(g):
        r = slice(at[i], at[i + 1])
        x, d, w = X[r].to(F64), dY[r].to(F64), W[i].to(F64)
        check(Y[r], x @ w.t(), x.abs() @ w.t().abs(), cols, 1)
        check(dX[r, cols:], d @ w, d.abs() @ w.abs(), rows, 1)
        check(dW[i], d.t() @ x, d.t().abs() @ x.abs(), max(1, lengths[i]), 1)


@pytest.mark.parametrize("lengths", [[1, 3, 2], [300, 1]], ids=str)
def test_adapters_on_views(lengths):
    b = Batch(lengths, [0, 1, -1][:len(lengths)], 2, 16, 72, 136, 0)
    big = torch.full((b.M, 3 * b.ldy), 7.0, dtype=torch.bfloat16, device="cuda")
    Y = big[:, b.ldy:b.ldy + 72]
    Y.copy_(b.Y0[:, :72])
    xx = torch.full((b.M, 2 * b.ldx), float("nan"), dtype=torch.bfloat16, device="cuda")
    xx[:, :136] = b.X[:, :136]
    B.mwu_adapters_add(2, 16, 72, 136, b.A[:, :16, :136], b.lda, 17 * b.lda, b.B[:, :72, :16], b.ldb, 73 * b.ldb, b.scale, len(lengths), b.off,
                       b.which, xx[:, :136], b.M, 2 * b.ldx, Y, Y, 3 * b.ldy, 0, b.st)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    assert bool((big[:, :b.ldy] == 7).all() & (big[:, b.ldy + 72:] == 7).all())
    got = b.Y0.clone()
    got[:, :72] = Y
    b.check(got, b.Y0, b.Y0)
