"""The bounded waits of the grouped products and of the adapters: a slot of the ring never fills (mwu_debug_rows_wait), the limit is about a
millisecond, the kernel comes back by itself with MWU_DEV_TIMEOUT, and the next call is right."""
import contextlib

import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_gpu_adapters import Batch
from test_gpu_grouped import F64, check, gen_of, new_status, normal, offsets_of

pytestmark = pytest.mark.gpu

LIMIT = 2_000_000


@contextlib.contextmanager
def waits(limit, slot=-1):
    B.mwu_debug_rows_wait(limit, slot)
    try:
        yield
        torch.cuda.synchronize()
    finally:
        B.mwu_debug_rows_wait(0, -1)


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("slot", [0, 3, 4])
@pytest.mark.parametrize("op", ["product", "dx", "dw"])
def test_grouped_products_come_back(op, slot, fp32):
    lengths, rows, cols = [200, 0, 1000, 77, 640], 1100, 1100      # a weight gradient's fourth stage is a group's last
    gen, at = gen_of(11), offsets_of(lengths)
    m, off = at[-1], torch.tensor(at, dtype=torch.int32, device="cuda")
    ld, n = 1104, len(lengths)
    W, X, dY = (torch.zeros(*s, ld, dtype=torch.bfloat16, device="cuda") for s in ((n, rows), (m,), (m,)))
    for t in (W, X, dY):
        t[..., :1100] = normal(gen, *t.shape[:-1], 1100, std=0.2)
    out = torch.zeros((n, rows, ld) if op == "dw" else (m, ld), dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")

    def call(st):
        if op == "dw":
            B.mwu_gemm_grouped_dw(n, rows, cols, off, dY, m, ld, X, ld, out, ld, rows * ld, fp32, 0, st)
        else:
            (B.mwu_gemm_grouped if op == "product" else B.mwu_gemm_grouped_dx)(n, rows, cols, W, ld, rows * ld, off, X, m, ld, out, ld, fp32, st)

    st = new_status()
    with waits(LIMIT, slot):
        call(st)
    assert int(st.item()) == B.MWU_DEV_TIMEOUT
    st.zero_()
    with waits(0):
        call(st)
    assert int(st.item()) == 0
    for g in range(n):
        r = slice(at[g], at[g + 1])
        if op == "dw":
            d, x = dY[r, :rows].to(F64).t(), X[r, :cols].to(F64)
            check(out[g, :, :cols], d @ x, d.abs() @ x.abs(), max(1, lengths[g]), fp32)
        else:
            x, w = X[r, :1100].to(F64), W[g, :, :1100].to(F64)
            w = w.t() if op == "product" else w
            check(out[r, :1100], x @ w, x.abs() @ w.abs(), 1100, fp32)


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("slot", [0, 1])
@pytest.mark.parametrize("rank", [16, 64, 128])
def test_adapters_come_back(rank, slot, fp32):
    b = Batch([700, 1, 0, 333, 40, 2], [0, 1, 2, -1, 2, 0], 3, rank, 1500, 1500, fp32)
    Y = torch.zeros_like(b.Y0)
    with waits(LIMIT, slot):
        b.run(b.Y0, Y)
    assert int(b.st.item()) == B.MWU_DEV_TIMEOUT
    b.st.zero_()
    before = Y.clone()
    with waits(0):
        b.run(b.Y0, Y)
    assert int(b.st.item()) == 0
    b.check(Y, b.Y0, before)


def test_a_limit_that_nothing_reaches_changes_nothing():
    b = Batch([700, 1], [0, 1], 2, 16, 520, 520, 0)
    Y, Z = torch.zeros_like(b.Y0), torch.zeros_like(b.Y0)
    b.run(b.Y0, Y)
    with waits(LIMIT, 1000):
        b.run(b.Y0, Z)
    assert int(b.st.item()) == 0 and torch.equal(Y, Z)


@pytest.mark.parametrize("lengths", [[(1 << 22) + 5], [1 << 22] + [16] * 73 + [13], [13] + [16] * 146 + [1 << 22, 5]], ids=lambda x: f"{len(x)} groups")
def test_a_group_may_take_longer_than_a_wait(lengths):
    """The limit is for one stage: a gradient of 4194304 rows takes 20 ms, several times the 2.5 ms set here, and the warp that zeroes
    foreign rows waits all through it, or through the tiles before its own."""
    gen, at, n = gen_of(12), offsets_of(lengths), len(lengths)
    m, off = at[-1], torch.tensor(at, dtype=torch.int32, device="cuda")
    dY, X, dW, st = normal(gen, m, 8), normal(gen, m, 8), torch.zeros(n, 8, 8, device="cuda"), new_status()
    with waits(5_000_000):
        B.mwu_gemm_grouped_dw(n, 8, 8, off, dY, m, 8, X, 8, dW, 8, 64, 1, 0, st)
    assert int(st.item()) == 0
    for g in range(n):
        d, x = dY[at[g]:at[g + 1]].to(F64).t(), X[at[g]:at[g + 1]].to(F64)
        check(dW[g], d @ x, d.abs() @ x.abs(), lengths[g], 1)
