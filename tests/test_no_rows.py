"""Grouped products and adapters on no rows: an empty tensor has no address, and none is asked for."""
import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_grouped_args import ADAPTERS, GRAD, INVALID, LINES

LATE = (B.MWU_ERR_CUDA, B.MWU_ERR_UNSUPPORTED_DEVICE)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the pointers are made up")
def test_no_address_is_needed_without_rows():
    for name in ("mwu_gemm_grouped", "mwu_gemm_grouped_dx"):
        assert getattr(B.lib(), name)(*dict(LINES, M=0, X=None, out=None).values()) in LATE
        assert getattr(B.lib(), name)(*dict(LINES, M=0, X=None, out=None, Wd=None).values()) == INVALID
        assert getattr(B.lib(), name)(*dict(LINES, M=1, out=None).values()) == INVALID
    assert B.lib().mwu_gemm_grouped_dw(*dict(GRAD, M=0, dY=None, X=None).values()) in LATE
    assert B.lib().mwu_gemm_grouped_dw(*dict(GRAD, M=0, dY=None, X=None, dW=None).values()) == INVALID
    assert B.lib().mwu_gemm_grouped_dw(*dict(GRAD, M=1, dY=None).values()) == INVALID
    assert B.lib().mwu_adapters_add(*dict(ADAPTERS, M=0, X=None, Y0=None, Y=None).values()) in LATE
    assert B.lib().mwu_adapters_add(*dict(ADAPTERS, segments=0, which=None).values()) in LATE
    assert B.lib().mwu_adapters_add(*dict(ADAPTERS, which=None).values()) == INVALID
    assert B.lib().mwu_adapters_add(*dict(ADAPTERS, M=1, Y=None).values()) == INVALID


@pytest.mark.gpu
def test_empty_tensors():
    groups, rows, cols, bf16 = 3, 24, 40, torch.bfloat16
    empty = lambda n, t=bf16: torch.empty(0, n, dtype=t, device="cuda")
    assert empty(cols).data_ptr() == 0
    W, off = torch.randn(groups, rows, cols, device="cuda").to(bf16), torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    for fp32 in (0, 1):
        t = torch.float32 if fp32 else bf16
        dW = torch.full((groups, rows, cols), 7.0, dtype=t, device="cuda")
        B.mwu_gemm_grouped(groups, rows, cols, W, cols, rows * cols, off, empty(cols), 0, cols, empty(rows, t), rows, fp32, st)
        B.mwu_gemm_grouped_dx(groups, rows, cols, W, cols, rows * cols, off, empty(rows), 0, rows, empty(cols, t), cols, fp32, st)
        if fp32:
            B.mwu_gemm_grouped_dw(groups, rows, cols, off, empty(rows), 0, rows, empty(cols), cols, dW, cols, rows * cols, 1, 1, st)
            torch.cuda.synchronize()
            assert bool((dW == 7).all())                    # nothing to add
        B.mwu_gemm_grouped_dw(groups, rows, cols, off, empty(rows), 0, rows, empty(cols), cols, dW, cols, rows * cols, fp32, 0, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0 and bool((dW == 0).all())
        A, Bm = torch.randn(2, 16, cols, device="cuda").to(bf16), torch.randn(2, rows, 16, device="cuda").to(bf16)
        which = torch.zeros(groups, dtype=torch.int32, device="cuda")
        for n, w, o in ((groups, which, off), (0, which[:0], off[:1])):
            B.mwu_adapters_add(2, 16, rows, cols, A, cols, 16 * cols, Bm, 16, rows * 16, None, n, o, w, empty(cols), 0, cols, empty(rows, t),
                               empty(rows, t), rows, fp32, st)
        x, y = torch.randn(5, cols, device="cuda").to(bf16), torch.full((5, rows), 7.0, dtype=t, device="cuda")
        B.mwu_adapters_add(2, 16, rows, cols, A, cols, 16 * cols, Bm, 16, rows * 16, None, 0, off[:1], which[:0], x, 5, cols, y, y, rows, fp32, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0 and bool((y == 7).all())
