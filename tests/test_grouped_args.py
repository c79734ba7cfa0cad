"""Arguments that the grouped products refuse, before any CUDA call (runs without a GPU)."""
import ctypes

import pytest

from paper_2106_08301_b200 import binding as B

P = ctypes.c_void_p(1 << 20)
INVALID, SHAPE, ALIGNMENT = B.MWU_ERR_INVALID_ARG, B.MWU_ERR_SHAPE, B.MWU_ERR_ALIGNMENT

LINES = dict(groups=4, rows=64, cols=128, Wd=P, ldw=128, w_stride=64 * 128, offsets=P, X=P, M=100, ldi=128, out=P, ldo=128, dtype=0,
             status=P, stream=None)
GRAD = dict(groups=4, rows=64, cols=128, offsets=P, dY=P, M=100, lddy=64, X=P, ldx=128, dW=P, lddw=128, stride=64 * 128, dtype=1,
            accumulate=0, status=P, stream=None)

COMMON = [(dict(M=-1), INVALID), (dict(offsets=None), INVALID), (dict(status=None), INVALID), (dict(X=None), INVALID),
          (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(groups=0), SHAPE), (dict(groups=-3), SHAPE),
          (dict(groups=B.MWU_MAX_GROUPS + 1), SHAPE), (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(M=2 ** 31), SHAPE),
          (dict(rows=B.MWU_MAX_GROUPED_SIDE + 1), SHAPE), (dict(offsets=ctypes.c_void_p((1 << 20) + 2)), ALIGNMENT),
          (dict(X=ctypes.c_void_p((1 << 20) + 8)), ALIGNMENT), (dict(status=ctypes.c_void_p((1 << 20) + 1)), ALIGNMENT)]


@pytest.mark.parametrize("name", ["mwu_gemm_grouped", "mwu_gemm_grouped_dx"])
@pytest.mark.parametrize("change,want", COMMON + [
    (dict(Wd=None), INVALID), (dict(out=None), INVALID), (dict(ldw=120), SHAPE), (dict(ldi=56), SHAPE), (dict(ldo=56), SHAPE),
    (dict(w_stride=64 * 128 - 8), SHAPE), (dict(w_stride=1 << 38), SHAPE), (dict(ldw=1 << 31, w_stride=1 << 37), SHAPE),
    (dict(ldw=132, w_stride=132 * 64), ALIGNMENT), (dict(w_stride=64 * 128 + 4), ALIGNMENT), (dict(ldi=132), ALIGNMENT),
    (dict(ldo=132), ALIGNMENT), (dict(ldo=130, dtype=1), ALIGNMENT), (dict(Wd=ctypes.c_void_p((1 << 20) + 8)), ALIGNMENT),
    (dict(out=ctypes.c_void_p((1 << 20) + 4)), ALIGNMENT)])
def test_products_refuse(name, change, want):
    assert getattr(B.lib(), name)(*dict(LINES, **change).values()) == want


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(dY=None), INVALID), (dict(dW=None), INVALID), (dict(accumulate=2), INVALID), (dict(accumulate=1, dtype=0), INVALID),
    (dict(lddy=56), SHAPE), (dict(ldx=120), SHAPE), (dict(lddw=124), SHAPE), (dict(stride=64 * 128 - 4), SHAPE),
    (dict(lddy=68), ALIGNMENT), (dict(ldx=132), ALIGNMENT), (dict(lddw=130, stride=130 * 64), ALIGNMENT),
    (dict(stride=64 * 128 + 2), ALIGNMENT), (dict(stride=64 * 128 + 4, dtype=0), ALIGNMENT),
    (dict(dW=ctypes.c_void_p((1 << 20) + 8)), ALIGNMENT), (dict(dY=ctypes.c_void_p((1 << 20) + 8)), ALIGNMENT)])
def test_weight_gradient_refuses(change, want):
    assert B.lib().mwu_gemm_grouped_dw(*dict(GRAD, **change).values()) == want


def test_what_is_allowed_reaches_the_device_check():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the pointers are made up")
    late = (B.MWU_ERR_CUDA, B.MWU_ERR_UNSUPPORTED_DEVICE)
    for name in ("mwu_gemm_grouped", "mwu_gemm_grouped_dx"):
        assert getattr(B.lib(), name)(*LINES.values()) in late
        assert getattr(B.lib(), name)(*dict(LINES, groups=B.MWU_MAX_GROUPS, M=1, dtype=1).values()) in late
    assert B.lib().mwu_gemm_grouped_dw(*GRAD.values()) in late
