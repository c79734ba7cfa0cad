"""mwu_adapters_add against the plain fp64 formula, segment by segment.

Tolerances, with S = sum_j |t_j| |b_nj| over T = X A^T of the same row, s = |scale|, and S2 the same with |t_j| replaced by
sum_k |x_k| |a_jk|.  T: sums of at most 512 products in a piece (cols / 8 in a cluster's CTA, or 512), within 512 / 8 * 2^-23 of
sum |x| |a| as for the grouped products, and cols / 512 + 8 roundings of 2^-24 where the pieces are added.  T enters the second
product as bf16 terms that leave out 2^-17 of it (two) or 2^-25 (three), which the next product adds up over rank / 16 steps a
term, within 2^-22 of the running magnitude each.  Y adds one rounding of 2^-24, and half a step of bf16, 2^-8, where it is bf16.
"""
import math
import random

import pytest
import torch

from paper_2106_08301_b200 import binding as B
from test_gpu_grouped import F64, gen_of, new_status, normal, offsets_of, padded, up8

pytestmark = pytest.mark.gpu


class Batch:
    def __init__(self, lengths, which, adapters, rank, rows, cols, fp32, seed=0, first=0, behind=0, pad=True, with_scale=True):
        gen = gen_of(seed + rank + rows + cols)
        self.lengths, self.which_list, self.n, self.k, self.r, self.adapters, self.fp32 = lengths, which, rows, cols, rank, adapters, fp32
        self.at = offsets_of(lengths, first)
        self.M = self.at[-1] + behind
        more = 8 if pad else 0
        self.lda, self.ldb, self.ldx, self.ldy = up8(cols) + more, up8(rank) + more, up8(cols) + 2 * more, up8(rows) + more
        nan = float("nan")
        self.A = torch.full((adapters, rank + 1, self.lda), nan, dtype=torch.bfloat16, device="cuda")
        self.A[:, :rank, :cols] = normal(gen, adapters, rank, cols, std=cols ** -0.5)
        self.B = torch.full((adapters, rows + 1, self.ldb), nan, dtype=torch.bfloat16, device="cuda")
        self.B[:, :rows, :rank] = normal(gen, adapters, rows, rank, std=0.3)
        self.scale = (torch.rand(adapters, generator=gen, device="cuda") * 2 - 0.7) if with_scale else None
        self.X = padded(gen, max(1, self.M), cols, self.ldx)
        if first:
            self.X[:first] = nan
        self.X[self.at[-1]:] = nan
        self.Y0 = torch.randn(max(1, self.M), self.ldy, generator=gen, device="cuda").to(torch.float32 if fp32 else torch.bfloat16)
        self.off = torch.tensor(self.at, dtype=torch.int32, device="cuda")
        self.which = torch.tensor(which if which else [0], dtype=torch.int32, device="cuda")
        self.st = new_status()

    def run(self, Y0, Y, stream=None, check=True):
        return B.mwu_adapters_add(self.adapters, self.r, self.n, self.k, self.A, self.lda, (self.r + 1) * self.lda, self.B, self.ldb,
                                  (self.n + 1) * self.ldb, self.scale, len(self.lengths), self.off, self.which, self.X, self.M, self.ldx,
                                  Y0, Y, self.ldy, self.fp32, self.st, stream, check)

    def check(self, Y, Y0, before):
        """Y against the formula on Y0 (None: zeros); what it must not touch against `before`."""
        n, k, r = self.n, self.k, self.r
        assert torch.equal(Y[:, n:], before[:, n:])
        assert torch.equal(Y[:self.at[0]], before[:self.at[0]]) and torch.equal(Y[self.at[-1]:], before[self.at[-1]:])
        for s, a in enumerate(self.which_list):
            rows = slice(self.at[s], self.at[s + 1])
            got = Y[rows, :n]
            base = torch.zeros_like(got) if Y0 is None else Y0[rows, :n]
            if a < 0:
                assert torch.equal(got, base)
                continue
            x, w, b = self.X[rows, :k].to(F64), self.A[a, :r, :k].to(F64), self.B[a, :n, :r].to(F64)
            sc = 1.0 if self.scale is None else float(self.scale[a])
            t = x @ w.t()
            ref = base.to(F64) + sc * (t @ b.t())
            S = abs(sc) * (t.abs() @ b.abs().t())
            S2 = abs(sc) * ((x.abs() @ w.abs().t()) @ b.abs().t())
            terms = 3 if self.fp32 else 2
            tol = (64 * 2.0 ** -23 + (k / 512 + 10) * 2.0 ** -24) * S2 + S * (2.0 ** (-17 if terms == 2 else -25) + (r / 16 + 1) * terms * 2.0 ** -22)
            tol = tol + (ref.abs() + base.to(F64).abs()) * 2.0 ** -23
            if not self.fp32:
                tol = tol + ref.abs() * 2.0 ** -8
            diff = (got.to(F64) - ref).abs()
            assert bool((diff <= tol + 1e-30).all()), (s, a, float((diff / (tol + 1e-30)).max()))


CASES = [       # lengths, adapters, rank, rows, cols
    ([1], 1, 1, 8, 8),
    ([1], 2, 16, 1, 1),
    ([1, 1, 1], 2, 8, 40, 100),
    ([1, 0, 2, 16, 17, 32, 0], 3, 16, 136, 264),
    ([3, 8, 9], 2, 5, 33, 31),
    ([7, 15], 2, 24, 1000, 1216),
    ([1] * 40, 5, 32, 520, 200),
    ([2, 30], 2, 57, 300, 77),
    ([4, 31], 2, 64, 257, 520),
    ([5, 20], 2, 128, 264, 300),
    ([9], 1, 100, 130, 4100),
    ([33], 1, 16, 64, 64),
    ([128], 1, 8, 8, 8),
    ([129, 1, 40], 2, 13, 70, 97),
    ([300, 33, 64], 3, 32, 200, 520),
    ([150, 500], 2, 64, 1000, 1216),
    ([257, 2, 131], 2, 96, 333, 200),
    ([1000], 1, 128, 520, 1040),
    ([32, 33, 1, 127, 0, 160], 4, 24, 1, 1),
    ([700, 5, 700, 1, 600], 3, 40, 136, 4104),
]


def which_of(lengths, adapters, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return [int(x) - 1 for x in torch.randint(0, adapters + 1, (len(lengths),), generator=g)]


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("lengths,adapters,rank,rows,cols", CASES)
def test_against_the_formula(lengths, adapters, rank, rows, cols, fp32):
    for seed, which in ((1, [s % adapters for s in range(len(lengths))]), (2, which_of(lengths, adapters, rank + rows))):
        b = Batch(lengths, which, adapters, rank, rows, cols, fp32, seed=seed, first=2, behind=5)
        before = torch.full_like(b.Y0, 777.0)
        Y = before.clone()
        b.run(b.Y0, Y)                                      # to another buffer
        torch.cuda.synchronize()
        assert int(b.st.item()) == 0
        b.check(Y, b.Y0, before)
        Z = b.Y0.clone()
        b.run(Z, Z)                                         # in place
        b.check(Z, b.Y0, b.Y0)
        assert all(torch.equal(Y[b.at[s]:b.at[s + 1], :rows], Z[b.at[s]:b.at[s + 1], :rows]) for s in range(len(lengths)))
        V = before.clone()
        b.run(None, V)                                      # nothing to add to
        b.check(V, None, before)
        assert int(b.st.item()) == 0


@pytest.mark.parametrize("seed", range(16))
def test_drawn_batches(seed):
    r = random.Random(seed)
    log = lambda lo, hi: int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))
    lengths = [1] * r.choice([0, log(1, 90)]) + [log(2, 1500) for _ in range(r.choice([0, 1, 3, 6]))] + [0] * r.choice([0, 2])
    r.shuffle(lengths)
    lengths = lengths or [1]
    adapters, rank, rows, cols = log(1, 20), r.choice([1, 7, 16, 31, 64, 65, 128, r.randrange(1, 129)]), log(1, 1100), log(1, 1500)
    b = Batch(lengths, [r.randrange(-1, adapters) for _ in lengths], adapters, rank, rows, cols, r.randrange(2), seed=seed, first=r.choice([0, 3]),
              behind=r.choice([0, 5]), pad=r.random() < 0.7, with_scale=r.random() < 0.7)
    before = torch.full_like(b.Y0, 777.0)
    Y = before.clone()
    b.run(b.Y0, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    b.check(Y, b.Y0, before)


def test_rows_of_one_adapter_all_over_the_batch():
    """A small batch is worked on adapter by adapter: many rows of one, in segments that lie apart, empty ones between."""
    lengths = [1, 0, 3, 1, 1, 0, 0, 20, 1, 1, 2, 1, 17, 1, 1, 1, 40, 1] + [1] * 60
    which = [(s * s) % 3 - 1 if s < 18 else 1 for s in range(len(lengths))]
    for fp32 in (0, 1):
        b = Batch(lengths, which, 2, 16, 264, 520, fp32)
        Z = b.Y0.clone()
        b.run(Z, Z)
        torch.cuda.synchronize()
        assert int(b.st.item()) == 0
        b.check(Z, b.Y0, b.Y0)


@pytest.mark.parametrize("lengths", [[1] * 257, [1] * 512, [1] * 513, [1] * 100 + [200] + [5] * 20 + [1] * 100, [1] * 1025, [32] * 16, [33] * 15 + [1],
                                     [31, 0, 33, 1] * 7 + [2] * 20], ids=lambda x: f"{len(x)}of{sum(x)}")
@pytest.mark.parametrize("adapters,fp32", [(1, 0), (7, 1), (40, 0)])
def test_batches_of_several_hundred_rows(lengths, adapters, fp32):
    """Rows of short segments are sorted by adapter up to 512 rows, beside the prompts; above, segment by segment."""
    r = random.Random(len(lengths) + adapters)
    b = Batch(lengths, [r.randrange(-1, adapters) for _ in lengths], adapters, 24, 72, 200, fp32, first=1 if sum(lengths) < 1024 else 0)
    Z = b.Y0.clone()
    b.run(Z, Z)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    # the formula for all rows at once, as in Batch.check
    seg = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths))
    a = torch.tensor(b.which_list)[seg].cuda()
    on, a = (a >= 0), a.clamp(min=0)
    rows = slice(b.at[0], b.at[-1])
    x, w, bm = b.X[rows, :200].to(F64), b.A[:, :24, :200].to(F64)[a], b.B[:, :72, :24].to(F64)[a]
    sc = b.scale.to(F64)[a] * on
    t = torch.einsum("mk,mrk->mr", x, w)
    base = b.Y0[rows, :72].to(F64)
    ref = base + sc[:, None] * torch.einsum("mr,mnr->mn", t, bm)
    S = sc.abs()[:, None] * torch.einsum("mr,mnr->mn", t.abs(), bm.abs())
    S2 = sc.abs()[:, None] * torch.einsum("mr,mnr->mn", torch.einsum("mk,mrk->mr", x.abs(), w.abs()), bm.abs())
    terms = 3 if fp32 else 2
    tol = (64 * 2.0 ** -23 + (200 / 512 + 10) * 2.0 ** -24) * S2 + S * (2.0 ** (-17 if terms == 2 else -25) + 2.5 * terms * 2.0 ** -22)
    tol = tol + (ref.abs() + base.abs()) * 2.0 ** -23 + (0 if fp32 else ref.abs() * 2.0 ** -8)
    got = Z[rows, :72]
    assert bool(((got.to(F64) - ref).abs() <= tol + 1e-30).all())
    assert torch.equal(got[~on], b.Y0[rows, :72][~on]) and torch.equal(Z[:, 72:], b.Y0[:, 72:]) and torch.equal(Z[:b.at[0]], b.Y0[:b.at[0]])


def test_without_scales_and_without_padding():
    for lengths in ([1, 1, 4], [200, 1]):
        b = Batch(lengths, [0] * len(lengths), 1, 16, 128, 256, 0, pad=False, with_scale=False)
        Y = torch.empty_like(b.Y0)
        b.run(b.Y0, Y)
        torch.cuda.synchronize()
        b.check(Y, b.Y0, Y)


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_request_holds_touches_no_other(bad, fp32):
    lengths, rank, rows, cols = [1, 150, 2, 40, 20, 128, 1], 24, 72, 136
    which = [0, 1, 2, 3, 4, 5, 6]
    for sick in range(7):
        b = Batch(lengths, which, 7, rank, rows, cols, fp32, seed=sick)
        b.X[b.at[sick]:b.at[sick + 1]] = bad
        b.A[sick], b.B[sick] = bad, bad
        Y = torch.empty_like(b.Y0)
        b.run(b.Y0, Y)
        torch.cuda.synchronize()
        assert not bool(torch.isfinite(Y[b.at[sick]:b.at[sick + 1], :rows]).any())
        b.which_list = [-1 if s == sick else s for s in range(7)]
        Y[b.at[sick]:b.at[sick + 1]] = b.Y0[b.at[sick]:b.at[sick + 1]]
        b.check(Y, b.Y0, Y)


@pytest.mark.parametrize("at,which", [([0, 5, 4, 9], [0, 0, 0]), ([-1, 3, 5, 9], [0, 0, 0]), ([0, 3, 5, 51], [0, 0, 0]), ([0, 3, 40, 50], [0, 2, 0]),
                                      ([0, 3, 40, 50], [0, -2, 0]), ([0, 3, 2 ** 31 - 1, 50], [0, 1, 0]), ([0, 0, 45, 45], [7, 0, 1])])
@pytest.mark.parametrize("M", [50, 20])
def test_lists_that_make_no_sense_write_nothing(at, which, M):
    if M == 20 and at[-1] <= 20:
        at = at[:1] + [20, 10, 20]
    b = Batch([M], [0], 2, 16, 40, 64, 1)
    b.lengths, b.off, b.which = [0, 0, 0], torch.tensor(at, dtype=torch.int32, device="cuda"), torch.tensor(which, dtype=torch.int32, device="cuda")
    Y = torch.full_like(b.Y0, 777.0)
    b.run(b.Y0, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == B.MWU_DEV_BOUNDS and bool((Y == 777).all())


def test_no_rows_and_no_segments():
    b = Batch([3], [0], 1, 16, 40, 64, 0)
    Y = torch.full_like(b.Y0, 777.0)
    b.lengths = []
    b.run(b.Y0, Y)
    b.lengths, b.M, b.off = [0, 0], 0, torch.zeros(3, dtype=torch.int32, device="cuda")
    b.which = torch.zeros(2, dtype=torch.int32, device="cuda")          # as long as the call says
    b.run(b.Y0, Y)
    b.M = 3
    b.run(b.Y0, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0 and bool((Y == 777).all())


def test_as_many_segments_as_there_may_be():
    n = B.MWU_MAX_SEGMENTS
    lengths = [1 if s % 3 else 0 for s in range(n)]
    lengths[5], lengths[4000] = 40, 300
    which = [(s * 7) % 12 - 1 for s in range(n)]
    which[5], which[4000] = 3, 4
    b = Batch(lengths, which, 11, 8, 24, 40, 1)
    Y = torch.empty_like(b.Y0)
    b.run(b.Y0, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    # row by row, all adapters at once
    seg = torch.repeat_interleave(torch.arange(n), torch.tensor(lengths))
    a = torch.tensor(which)[seg].cuda()
    on = (a >= 0).to(F64)
    a = a.clamp(min=0)
    x, w, bm = b.X[:b.M, :40].to(F64), b.A[:, :8, :40].to(F64)[a], b.B[:, :24, :8].to(F64)[a]
    t = torch.einsum("mk,mrk->mr", x, w)
    ref = b.Y0[:, :24].to(F64) + (on * b.scale[a].to(F64))[:, None] * torch.einsum("mr,mnr->mn", t, bm)
    # (40 + 8 products: 2^-18 of their magnitude, which stays below 100, is beyond what the formula above allows)
    assert float((Y[:, :24].to(F64) - ref).abs().max()) < 100 * 2.0 ** -18


def test_the_same_bits_again_on_two_streams_and_in_a_graph():
    a = Batch([1] * 30 + [100, 700], [s % 4 for s in range(32)], 4, 16, 264, 520, 0, seed=1)
    b = Batch([400, 2, 1, 1, 1, 900], [0, 1, 2, 0, 1, 2], 3, 64, 392, 328, 1, seed=2)
    outs = [torch.empty_like(x.Y0) for x in (a, b)]
    for x, y in zip((a, b), outs):
        x.run(x.Y0, y)
    torch.cuda.synchronize()
    want = [y[:, :x.n].clone() for x, y in zip((a, b), outs)]          # (behind it is whatever the buffer held, NaN perhaps)
    for x, y in zip((a, b), outs):
        x.check(y, x.Y0, y)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for x, y, s in zip((a, b), outs, streams):
            x.run(x.Y0, y, s)
    torch.cuda.synchronize()
    assert int(a.st.item()) == 0 and int(b.st.item()) == 0
    assert all(torch.equal(y[:, :x.n], w) for x, y, w in zip((a, b), outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, y in zip((a, b), outs):
            x.run(x.Y0, y)
    for y in outs:
        y.zero_()
    a.which.copy_(torch.tensor([(s + 1) % 4 for s in range(32)], dtype=torch.int32))      # read on the device
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    a.which_list = [(s + 1) % 4 for s in range(32)]
    a.check(outs[0], a.Y0, outs[0])
    assert torch.equal(outs[1][:, :b.n], want[1])


def test_what_follows_sees_the_rows_of_both_kernels():
    """Prompts and tokens are worked on by two kernels at the same time; the next call on the stream comes behind both."""
    b = Batch([1, 2000, 1, 1, 1500, 3], [0, 1, 0, 1, 0, 1], 2, 16, 520, 1040, 0, pad=False)
    for _ in range(30):
        Y = torch.full_like(b.Y0, float("nan"))
        b.run(b.Y0, Y)
        Z = Y.clone()
        assert not bool(torch.isnan(Z).any())
    b.check(Z, b.Y0, Z)


def test_positions_beyond_32_bits():
    rows, cols, rank = 64, 64, 16
    b = Batch([70000], [0], 1, rank, rows, cols, 0, pad=False)
    m, ld = 70000, 32768
    X = torch.zeros(m, ld, dtype=torch.bfloat16, device="cuda")
    X[:, :cols] = b.X[:, :cols]
    Y = torch.full((m, ld), 777.0, dtype=torch.bfloat16, device="cuda")
    at = [0, 100, m - 301, m - 1, m]
    off, which, st = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (at, [0, 0, 0, 0], [0]))
    B.mwu_adapters_add(1, rank, rows, cols, b.A, b.lda, (rank + 1) * b.lda, b.B, b.ldb, (rows + 1) * b.ldb, b.scale, 4, off, which, X, m, ld,
                       None, Y, ld, 0, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and bool((Y[-400:, rows:] == 777).all())
    c = Batch([m], [0], 1, rank, rows, cols, 0, pad=False)
    c.X, c.A, c.B, c.scale = b.X, b.A, b.B, b.scale
    c.check(Y[:, :rows].contiguous(), None, Y[:, :rows].contiguous())


def test_beside_a_compressed_projection():
    """As it is used: one packed layer for all requests, a prompt and single tokens with adapters of their own, in place."""
    rows, cols, m = 512, 256, 400
    gen = gen_of(77)
    W = torch.randn(rows, cols, generator=gen, device="cuda") * 0.02
    blocks = rows * cols // 8
    desc = B.make_desc(rows, cols, 8, blocks // 2, blocks // 4)
    bufs = B.ProjectionBuffers(desc)
    bufs.project(W)
    packed = bufs.pack(W)
    Wd = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    B.mwu_decode(desc, packed, Wd, cols, bufs.dev_status)
    b = Batch([300, 1, 1, 0, 98], [0, 1, -1, 2, 2], 3, 16, rows, cols, 1, pad=False)
    Y = torch.empty(m, rows, device="cuda")
    for _ in range(3):
        B.mwu_gemm(desc, packed, b.X, m, cols, Y, rows, 1, bufs.dev_status)
        base = Y.clone()
        B.mwu_gemm(desc, packed, b.X, m, cols, Y, rows, 1, bufs.dev_status)
        b.run(Y, Y)
        B.mwu_gemm(desc, packed, b.X, m, cols, base, rows, 1, bufs.dev_status)
    torch.cuda.synchronize()
    assert int(bufs.dev_status.item()) == 0 and int(b.st.item()) == 0
    b.check(Y, base, Y)
    ref = b.X.to(F64) @ Wd.to(F64).t()
    assert float((base.to(F64) - ref).norm() / ref.norm()) <= 1e-5


def test_training_an_adapter():
    """Gradients of X, A and B by grouped products, against those of the formula and against autograd in fp64.

    T and dT are rounded to bf16 (2^-8 of each of their entries), and so are the results (2^-8 of them)."""
    lengths, rank, rows, cols = [70, 0, 33, 130], 16, 200, 136
    b = Batch(lengths, [0, 1, 2, 3], 4, rank, rows, cols, 0, pad=False, with_scale=False)
    gen, g, m = gen_of(3), 4, b.M
    A, Bm = b.A[:, :rank].contiguous(), b.B[:, :rows].contiguous()
    dY = normal(gen, m, rows)
    T, dT = (torch.empty(m, rank, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dX, dA, dB = torch.empty_like(b.X), torch.empty_like(A), torch.empty_like(Bm)
    st, off = new_status(), b.off
    B.mwu_gemm_grouped(g, rank, cols, A, cols, rank * cols, off, b.X, m, cols, T, rank, 0, st)
    B.mwu_gemm_grouped_dx(g, rows, rank, Bm, rank, rows * rank, off, dY, m, rows, dT, rank, 0, st)
    B.mwu_gemm_grouped_dx(g, rank, cols, A, cols, rank * cols, off, dT, m, rank, dX, cols, 0, st)
    B.mwu_gemm_grouped_dw(g, rank, cols, off, dT, m, rank, b.X, cols, dA, cols, rank * cols, 0, 0, st)
    B.mwu_gemm_grouped_dw(g, rows, rank, off, dY, m, rows, T, rank, dB, rank, rows * rank, 0, 0, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for s in range(g):
        r = slice(b.at[s], b.at[s + 1])
        x, a, bb = (v.to(F64).requires_grad_() for v in (b.X[r], A[s], Bm[s]))
        d = dY[r].to(F64)
        y = (x @ a.t()) @ bb.t()
        y.backward(d)
        by_autograd = (x.grad, a.grad, bb.grad)
        t, dt = (x @ a.t()).detach().abs(), (d @ bb).detach().abs()
        # 1.01: the roundings of the sums themselves, 2^-16 of a magnitude that is below 2^8 times the result's own tolerance
        slack = (256 / 8 + 8) * 2.0 ** -23
        x, a, bb = x.detach(), a.detach(), bb.detach()
        ax, aa, ab, ad = x.abs(), a.abs(), bb.abs(), d.abs()
        for (got, ref, low, mag), auto in zip(((dX[r], (d @ bb) @ a, dt @ aa, (ad @ ab) @ aa), (dA[s], (d @ bb).t() @ x, dt.t() @ ax, (ad @ ab).t() @ ax),
                                   (dB[s], d.t() @ (x @ a.t()), ad.t() @ t, ad.t() @ (ax @ aa.t()))), by_autograd):
            assert bool(((ref - auto).abs() <= 1e-12 * (mag + 1e-30)).all())
            tol = 1.01 * 2.0 ** -8 * (low + ref.abs()) + 2 * slack * mag + 1e-30
            assert bool(((got.to(F64) - ref).abs() <= tol).all())
