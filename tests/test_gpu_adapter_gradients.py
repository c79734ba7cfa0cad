"""An adapter's gradients in fp32 by grouped products: X A^T and dY B as two bf16 terms each instead of one.

A term pair leaves out 2^-17 of each entry of T = X A^T and dT = dY B (one bf16 alone: 2^-8), every fp32 sum of up to 256 products is
within 256 / 8 + 8 units of 2^-23 of its magnitude, T's and the result's, and results round by 2^-24."""
import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_gpu_adapters import Batch
from test_gpu_grouped import F64, gen_of, new_status, normal

pytestmark = pytest.mark.gpu


def two_terms(t):
    """[t1 t2] with t1 + t2 = t but for 2^-17 of it, side by side."""
    hi = t.to(torch.bfloat16)
    return torch.cat([hi, (t - hi.float()).to(torch.bfloat16)], 1)


def test_training_an_adapter_in_more_bits():
    lengths, rank, rows, cols = [70, 0, 33, 130], 16, 200, 136
    b = Batch(lengths, [0, 1, 2, 3], 4, rank, rows, cols, 0, pad=False, with_scale=False)
    gen, g, m = gen_of(3), 4, b.M
    A, Bm = b.A[:, :rank].contiguous(), b.B[:, :rows].contiguous()
    AA = torch.cat([A, A], 1)                               # [groups][2 rank][cols]
    dY, st, off = normal(gen, m, rows), new_status(), b.off
    T, dT = (torch.empty(m, rank, device="cuda") for _ in range(2))
    dX, dA, dB = torch.empty(m, cols, device="cuda"), torch.empty(g, rank, cols, device="cuda"), torch.empty(g, rows, rank, device="cuda")
    B.mwu_gemm_grouped(g, rank, cols, A, cols, rank * cols, off, b.X, m, cols, T, rank, 1, st)
    B.mwu_gemm_grouped_dx(g, rows, rank, Bm, rank, rows * rank, off, dY, m, rows, dT, rank, 1, st)
    T2, dT2 = two_terms(T), two_terms(dT)
    B.mwu_gemm_grouped_dx(g, 2 * rank, cols, AA, cols, 2 * rank * cols, off, dT2, m, 2 * rank, dX, cols, 1, st)
    for term in range(2):
        lo = slice(term * rank, (term + 1) * rank)
        B.mwu_gemm_grouped_dw(g, rank, cols, off, dT2[:, lo], m, 2 * rank, b.X, cols, dA, cols, rank * cols, 1, term, st)
        B.mwu_gemm_grouped_dw(g, rows, rank, off, dY, m, rows, T2[:, lo], 2 * rank, dB, rank, rows * rank, 1, term, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    far = 0.0
    for s in range(g):
        r = slice(b.at[s], b.at[s + 1])
        x, a, bb, d = b.X[r].to(F64), A[s].to(F64), Bm[s].to(F64), dY[r].to(F64)
        t, dt = x @ a.t(), d @ bb
        slack = (256 / 8 + 8) * 2.0 ** -23
        ax, aa, ab, ad = x.abs(), a.abs(), bb.abs(), d.abs()
        for got, ref, low, mag in ((dX[r], dt @ a, dt.abs() @ aa, (ad @ ab) @ aa), (dA[s], dt.t() @ x, dt.abs().t() @ ax, (ad @ ab).t() @ ax),
                                   (dB[s], d.t() @ t, ad.t() @ t.abs(), ad.t() @ (ax @ aa.t()))):
            tol = 2.0 ** -17 * low + 2 * slack * mag + 2.0 ** -24 * ref.abs()
            assert bool(((got.to(F64) - ref).abs() <= tol).all())
            if ref.numel() and float(ref.norm()):
                far = max(far, float((got.to(F64) - ref).norm() / ref.norm()))
    assert far < 2.0 ** -16                                 # entries of T off by 2^-17 at most; one term alone shows 1e-3 and more
