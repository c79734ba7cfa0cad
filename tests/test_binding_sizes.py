"""The binding of the grouped products and of the adapters checks what a call reaches against the tensors that it is given (on the CPU:
tensors of the `meta` kind in the place of the device's, and a library that only says it was called)."""
import pytest
import torch

from paper_2106_08301_b200 import binding as B

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Library:
    def __getattr__(self, name):
        return lambda *a: B.MWU_OK


@pytest.fixture(autouse=True)
def no_device(monkeypatch):
    monkeypatch.setattr(B, "lib", lambda: Library())
    monkeypatch.setattr(B, "_get_device", lambda: -1)           # what a tensor of no CUDA device answers
    monkeypatch.setattr(B, "_stream_on", lambda stream, device: 0)
    monkeypatch.setattr(B, "_data_ptr", lambda t: 1 << 20)


def new(*shape, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="meta")


G, N, K, M = 3, 24, 40, 9
PRODUCT = dict(groups=G, rows=N, cols=K, Wd=new(G, N, K), ldw=K, w_stride=N * K, offsets=new(G + 1, dtype=I32), X=new(M, K), M=M, ldx=K,
               Y=new(M, N, dtype=F32), ldy=N, y_dtype=1, dev_status=new(1, dtype=I32))
DX = dict(groups=G, rows=N, cols=K, Wd=new(G, N, K), ldw=K, w_stride=N * K, offsets=new(G + 1, dtype=I32), dY=new(M, N), M=M, lddy=N,
          dX=new(M, K), lddx=K, dx_dtype=0, dev_status=new(1, dtype=I32))
DW = dict(groups=G, rows=N, cols=K, offsets=new(G + 1, dtype=I32), dY=new(M, N), M=M, lddy=N, X=new(M, K), ldx=K,
          dW=new(G, N, K, dtype=F32), lddw=K, dw_stride=N * K, dw_dtype=1, accumulate=0, dev_status=new(1, dtype=I32))
ADAPTERS = dict(adapters=2, rank=16, rows=N, cols=K, A=new(2, 16, K), lda=K, a_stride=16 * K, Bm=new(2, N, 16), ldb=16, b_stride=16 * N,
                scale=new(2, dtype=F32), segments=3, offsets=new(4, dtype=I32), which=new(3, dtype=I32), X=new(M, K), M=M, ldx=K, Y0=new(M, N),
                Y=new(M, N), ldy=N, y_dtype=0, dev_status=new(1, dtype=I32))
CALLS = {"mwu_gemm_grouped": PRODUCT, "mwu_gemm_grouped_dx": DX, "mwu_gemm_grouped_dw": DW, "mwu_adapters_add": ADAPTERS}
TENSORS = [(name, key) for name, args in CALLS.items() for key, t in args.items() if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("name", CALLS)
def test_what_is_just_large_enough_is_taken(name):
    assert getattr(B, name)(**CALLS[name]) == B.MWU_OK


@pytest.mark.parametrize("name,key", TENSORS)
def test_a_tensor_that_is_too_small_is_refused(name, key):
    t = CALLS[name][key]
    with pytest.raises(ValueError):
        getattr(B, name)(**{**CALLS[name], key: t.flatten()[:-1]})
    if t.dim() > 1:                                             # whatever its shape, it is the reach that counts
        assert getattr(B, name)(**{**CALLS[name], key: t.flatten()}) == B.MWU_OK


@pytest.mark.parametrize("name,change", [("mwu_gemm_grouped", dict(groups=4)), ("mwu_gemm_grouped", dict(M=10)), ("mwu_gemm_grouped", dict(ldx=48)),
                                         ("mwu_gemm_grouped", dict(w_stride=N * K + 8)), ("mwu_gemm_grouped_dx", dict(lddx=48)),
                                         ("mwu_gemm_grouped_dx", dict(rows=25)), ("mwu_gemm_grouped_dw", dict(lddw=44)),
                                         ("mwu_gemm_grouped_dw", dict(dw_stride=N * K + 4)), ("mwu_gemm_grouped_dw", dict(M=10)),
                                         ("mwu_adapters_add", dict(segments=4)), ("mwu_adapters_add", dict(adapters=3)),
                                         ("mwu_adapters_add", dict(rank=17)), ("mwu_adapters_add", dict(ldy=32)), ("mwu_adapters_add", dict(M=10))])
def test_sizes_beyond_the_tensors_are_refused(name, change):
    with pytest.raises(ValueError):
        getattr(B, name)(**{**CALLS[name], **change})


def test_no_rows_reach_nothing():
    assert B.mwu_gemm_grouped(**{**PRODUCT, "M": 0, "X": new(0, K), "Y": new(0, N, dtype=F32)}) == B.MWU_OK
    assert B.mwu_adapters_add(**{**ADAPTERS, "M": 0, "X": new(0, K), "Y": new(0, N), "Y0": None, "scale": None}) == B.MWU_OK


def wide(*shape, dtype=BF16, more=8):
    """A view of the first columns of a wider buffer."""
    return new(*shape[:-1], shape[-1] + more, dtype=dtype)[..., :shape[-1]]


def test_views_with_contiguous_rows_are_taken():
    assert B.mwu_gemm_grouped(**{**PRODUCT, "Wd": wide(G, N, K), "ldw": K + 8, "w_stride": N * (K + 8), "X": wide(M, K), "ldx": K + 8,
                                 "Y": wide(M, N, dtype=F32), "ldy": N + 8}) == B.MWU_OK
    assert B.mwu_gemm_grouped_dw(**{**DW, "dW": new(G, 2, N, K, dtype=F32)[:, 1], "dw_stride": 2 * N * K, "dY": wide(M, N), "lddy": N + 8}) == B.MWU_OK
    assert B.mwu_adapters_add(**{**ADAPTERS, "X": wide(M, K), "ldx": K + 8, "Y": wide(M, N), "Y0": None, "ldy": N + 8}) == B.MWU_OK


@pytest.mark.parametrize("change", [dict(X=wide(M, K)[:-1], ldx=K + 8), dict(X=wide(M, K), ldx=K + 16), dict(X=new(K, M).t()),
                                    dict(X=new(1, K).expand(M, K)), dict(X=new(M, 2 * K)[:, ::2], ldx=2 * K), dict(offsets=new(2 * G + 2, dtype=I32)[::2]),
                                    dict(X=wide(M, K, dtype=F32), ldx=K + 8), dict(Y=new(N, M, dtype=F32).t())])
def test_other_views_are_refused(change):
    with pytest.raises(ValueError):
        B.mwu_gemm_grouped(**{**PRODUCT, **change})
