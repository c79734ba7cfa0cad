"""Arguments that the grouped products and the adapters refuse, before any CUDA call (runs without a GPU)."""
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


ADAPTERS = dict(adapters=4, rank=16, rows=64, cols=128, A=P, lda=128, a_stride=16 * 128, B=P, ldb=16, b_stride=64 * 16, scale=P, segments=3,
                offsets=P, which=P, X=P, M=100, ldx=128, Y0=P, Y=P, ldy=64, dtype=0, status=P, stream=None)
ODD = ctypes.c_void_p((1 << 20) + 8)


@pytest.mark.parametrize("change,want", [
    (dict(A=None), INVALID), (dict(B=None), INVALID), (dict(offsets=None), INVALID), (dict(which=None), INVALID), (dict(X=None), INVALID),
    (dict(Y=None), INVALID), (dict(status=None), INVALID), (dict(M=-1), INVALID), (dict(dtype=2), INVALID),
    (dict(adapters=0), SHAPE), (dict(adapters=1 << 31), SHAPE), (dict(segments=-1), SHAPE), (dict(segments=B.MWU_MAX_SEGMENTS + 1), SHAPE),
    (dict(rank=0), SHAPE), (dict(rank=B.MWU_MAX_RANK + 1, ldb=256, a_stride=1 << 20, b_stride=1 << 20), SHAPE), (dict(rows=0), SHAPE),
    (dict(cols=0), SHAPE), (dict(rows=B.MWU_MAX_GROUPED_SIDE + 1), SHAPE), (dict(M=2 ** 31), SHAPE), (dict(lda=120), SHAPE), (dict(ldb=8), SHAPE),
    (dict(ldx=120), SHAPE), (dict(ldy=56), SHAPE), (dict(a_stride=16 * 128 - 8), SHAPE), (dict(b_stride=64 * 16 - 8), SHAPE),
    (dict(lda=132, a_stride=16 * 132), ALIGNMENT), (dict(ldb=20, b_stride=64 * 20), ALIGNMENT), (dict(ldx=132), ALIGNMENT),
    (dict(a_stride=16 * 128 + 4), ALIGNMENT), (dict(b_stride=64 * 16 + 4), ALIGNMENT), (dict(ldy=68), ALIGNMENT), (dict(ldy=66, dtype=1), ALIGNMENT),
    (dict(A=ODD), ALIGNMENT), (dict(B=ODD), ALIGNMENT), (dict(X=ODD), ALIGNMENT), (dict(Y0=ODD), ALIGNMENT), (dict(Y=ODD), ALIGNMENT),
    (dict(scale=ctypes.c_void_p((1 << 20) + 2)), ALIGNMENT), (dict(which=ctypes.c_void_p((1 << 20) + 2)), ALIGNMENT)])
def test_adapters_refuse(change, want):
    assert B.lib().mwu_adapters_add(*dict(ADAPTERS, **change).values()) == want


def test_adapters_that_are_allowed_reach_the_device_check():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the pointers are made up")
    for change in (dict(), dict(Y0=None, scale=None), dict(rank=B.MWU_MAX_RANK, ldb=128, a_stride=128 * 128, b_stride=64 * 128), dict(dtype=1, ldy=68)):
        assert B.lib().mwu_adapters_add(*dict(ADAPTERS, **change).values()) in (B.MWU_ERR_CUDA, B.MWU_ERR_UNSUPPORTED_DEVICE)
