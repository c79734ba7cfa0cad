"""Grouped products and their gradients (mwu_gemm_grouped, _dx, _dw) against plain fp64 products, group by group.

Tolerances.  A tensor-core step adds 16 products to an fp32 accumulator and may be off by two units in the last place of the
running magnitude, at most 2^-22 of S = sum |a| |b|; K products take K / 16 steps, so a sum is within K / 8 * 2^-23 * S,
with K the length of a piece (512) where the result is fp32, and the pieces are added with K / 512 roundings of 2^-24.
A bf16 result adds half a step of it, 2^-8.
"""
import math
import random

import pytest
import torch

from paper_2106_08301_b200 import binding as B

pytestmark = pytest.mark.gpu

F64 = torch.float64


def offsets_of(lengths, first=0):
    at = [first]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def normal(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(torch.bfloat16)


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def padded(gen, rows, cols, ld, std=1.0):
    """A [rows][ld] buffer whose padding is NaN."""
    t = torch.full((rows, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
    t[:, :cols] = normal(gen, rows, cols, std=std)
    return t


def check(got, ref, mag, k, fp32):
    """got against the fp64 result ref, whose terms add up to mag in magnitude."""
    piece = min(k, 512) if fp32 else k
    tol = (piece / 8 + 8) * 2.0 ** -23 * mag
    if fp32:
        tol = tol + (k / 512 + 1) * 2.0 ** -24 * mag
    else:
        tol = tol + ref.abs() * 2.0 ** -8 + 2.0 ** -126
    diff = (got.to(F64) - ref).abs()
    assert bool((diff <= tol).all()), float((diff / (tol + 1e-300)).max())


def up8(n):
    return (n + 7) // 8 * 8


def new_status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def sentinel(rows, ld, dtype):
    return torch.full((rows, ld), 777.0, dtype=dtype, device="cuda")


SHAPES = [                                      # lengths, rows, cols
    ([1], 8, 8),
    ([3, 0, 1, 5], 1, 1),
    ([2, 31, 32, 33], 37, 50),
    ([0, 0, 0], 64, 64),
    ([255, 256, 257, 0, 1], 130, 200),
    ([600, 1, 0, 77], 256, 512),
    ([17, 300, 513], 300, 1216),
    ([1024, 5], 1000, 520),
    ([129], 520, 4100),
]


@pytest.mark.parametrize("fp32", [0, 1])
@pytest.mark.parametrize("dx", [False, True])
@pytest.mark.parametrize("lengths,rows,cols", SHAPES)
def test_product_and_input_gradient(lengths, rows, cols, dx, fp32):
    gen = gen_of(sum(lengths) + rows + cols)
    groups, first, behind = len(lengths), 3, 9
    at = offsets_of(lengths, first)
    M = at[-1] + behind
    red, feat = (rows, cols) if dx else (cols, rows)
    ldw, ldi, ldo = up8(cols) + 8, up8(red) + 16, up8(feat) + 8
    w_stride = (rows + 2) * ldw
    W = torch.full((groups, rows + 2, ldw), float("nan"), dtype=torch.bfloat16, device="cuda")
    W[:, :rows, :cols] = normal(gen, groups, rows, cols, std=0.05)
    X = padded(gen, M, red, ldi)
    X[:first] = float("nan")                    # rows of no group
    X[at[-1]:] = float("inf")
    Y = sentinel(M, ldo, torch.float32 if fp32 else torch.bfloat16)
    st = new_status()
    off = torch.tensor(at, dtype=torch.int32, device="cuda")
    call = B.mwu_gemm_grouped_dx if dx else B.mwu_gemm_grouped
    call(groups, rows, cols, W, ldw, w_stride, off, X, M, ldi, Y, ldo, fp32, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert bool((Y[:first] == 777).all()) and bool((Y[at[-1]:] == 777).all()) and bool((Y[:, feat:] == 777).all())
    for g in range(groups):
        x = X[at[g]:at[g + 1], :red].to(F64)
        w = W[g, :rows, :cols].to(F64)
        w = w if dx else w.t()
        check(Y[at[g]:at[g + 1], :feat], x @ w, x.abs() @ w.abs(), red, fp32)


@pytest.mark.parametrize("mode", ["bf16", "fp32", "accumulate"])
@pytest.mark.parametrize("lengths,rows,cols", SHAPES + [([16, 48, 64, 80, 63, 65], 24, 40), ([1040, 1], 257, 300)])
def test_weight_gradient(lengths, rows, cols, mode):
    gen = gen_of(sum(lengths) + rows + cols + 1)
    groups, first, behind = len(lengths), 5, 11
    at = offsets_of(lengths, first)
    M = at[-1] + behind
    lddy, ldx, lddw = up8(rows) + 8, up8(cols) + 16, up8(cols) + 8
    dw_stride = (rows + 1) * lddw
    dY, X = padded(gen, M, rows, lddy), padded(gen, M, cols, ldx)
    for t in (dY, X):
        t[:first] = float("nan")
        t[at[-1]:] = float("nan")
    fp32 = mode != "bf16"
    dW = torch.full((groups, rows + 1, lddw), 777.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    if mode == "accumulate":
        dW[:, :rows, :cols] = torch.randn(groups, rows, cols, generator=gen, device="cuda")
    before = dW.clone()
    st = new_status()
    off = torch.tensor(at, dtype=torch.int32, device="cuda")
    B.mwu_gemm_grouped_dw(groups, rows, cols, off, dY, M, lddy, X, ldx, dW, lddw, dw_stride, int(fp32), int(mode == "accumulate"), st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert bool((dW[:, rows:] == 777).all()) and bool((dW[:, :, cols:] == 777).all())
    for g in range(groups):
        d, x = dY[at[g]:at[g + 1], :rows].to(F64), X[at[g]:at[g + 1], :cols].to(F64)
        ref, mag = d.t() @ x, d.abs().t() @ x.abs()
        if mode == "accumulate":
            ref, mag = ref + before[g, :rows, :cols].to(F64), mag + before[g, :rows, :cols].abs().to(F64)
        if lengths[g] == 0:
            assert torch.equal(dW[g, :rows, :cols], before[g, :rows, :cols] if mode == "accumulate" else torch.zeros_like(before[g, :rows, :cols]))
        else:
            check(dW[g, :rows, :cols], ref, mag, lengths[g], fp32)


@pytest.mark.parametrize("seed", range(16))
def test_drawn_sizes(seed):
    """Sizes between the listed ones: every height of tile, sides as long as a rank, few and many rows to a group."""
    r = random.Random(seed)
    log = lambda lo, hi: int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))
    groups, m = log(1, 40), log(1, 6000)
    rows, cols = ([log(1, 900), r.choice([8, 16, 24, 64, 72, 128])] if r.random() < 0.5 else [log(1, 700), log(1, 1100)])
    if r.random() < 0.5:
        rows, cols = cols, rows
    gen = gen_of(1000 + seed)
    which = torch.sort(torch.randint(groups, (m,), generator=gen, device="cuda"))[0]
    off = torch.searchsorted(which, torch.arange(groups + 1, device="cuda")).to(torch.int32)
    at, st = off.tolist(), new_status()
    ldw, ldx, ldy = up8(cols), up8(cols), up8(rows)
    W, X, dY = padded(gen, groups * rows, cols, ldw, std=0.1), padded(gen, m, cols, ldx), padded(gen, m, rows, ldy)
    for fp32 in (0, 1):
        t = torch.float32 if fp32 else torch.bfloat16
        Y, dX, dW = sentinel(m, ldy, t), sentinel(m, ldx, t), sentinel(groups * rows, ldw, t)
        B.mwu_gemm_grouped(groups, rows, cols, W, ldw, rows * ldw, off, X, m, ldx, Y, ldy, fp32, st)
        B.mwu_gemm_grouped_dx(groups, rows, cols, W, ldw, rows * ldw, off, dY, m, ldy, dX, ldx, fp32, st)
        B.mwu_gemm_grouped_dw(groups, rows, cols, off, dY, m, ldy, X, ldx, dW, ldw, rows * ldw, fp32, 0, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        assert bool((Y[:, rows:] == 777).all() & (dX[:, cols:] == 777).all() & (dW[:, cols:] == 777).all())
        for g in range(groups):
            rng, mine = slice(at[g], at[g + 1]), slice(g * rows, (g + 1) * rows)
            x, d, w = X[rng, :cols].to(F64), dY[rng, :rows].to(F64), W[mine, :cols].to(F64)
            check(Y[rng, :rows], x @ w.t(), x.abs() @ w.t().abs(), cols, fp32)
            check(dX[rng, :cols], d @ w, d.abs() @ w.abs(), rows, fp32)
            check(dW[mine, :cols], d.t() @ x, d.t().abs() @ x.abs(), max(1, at[g + 1] - at[g]), fp32)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_one_group_holds_touches_no_other(bad):
    lengths, rows, cols = [21, 40, 1, 130, 7], 72, 136
    at, gen = offsets_of(lengths), gen_of(5)
    M, off = at[-1], torch.tensor(at, dtype=torch.int32, device="cuda")
    for sick in range(len(lengths)):
        W, X, dY = normal(gen, 5, rows, cols, std=0.1), normal(gen, M, cols), normal(gen, M, rows)
        W[sick] = bad
        X[at[sick]:at[sick + 1]] = bad
        dY[at[sick]:at[sick + 1]] = bad
        Y, dX = (torch.empty(M, n, device="cuda") for n in (rows, cols))
        dW, st = torch.empty(5, rows, cols, device="cuda"), new_status()
        B.mwu_gemm_grouped(5, rows, cols, W, cols, rows * cols, off, X, M, cols, Y, rows, 1, st)
        B.mwu_gemm_grouped_dx(5, rows, cols, W, cols, rows * cols, off, dY, M, rows, dX, cols, 1, st)
        B.mwu_gemm_grouped_dw(5, rows, cols, off, dY, M, rows, X, cols, dW, cols, rows * cols, 1, 0, st)
        torch.cuda.synchronize()
        for g in range(5):
            rng = slice(at[g], at[g + 1])
            if g == sick:
                assert not bool(torch.isfinite(Y[rng]).any() | torch.isfinite(dX[rng]).any() | torch.isfinite(dW[g]).any())
                continue
            x, d, w = X[rng].to(F64), dY[rng].to(F64), W[g].to(F64)
            check(Y[rng], x @ w.t(), x.abs() @ w.t().abs(), cols, 1)
            check(dX[rng], d @ w, d.abs() @ w.abs(), rows, 1)
            check(dW[g], d.t() @ x, d.t().abs() @ x.abs(), lengths[g], 1)


@pytest.mark.parametrize("m", [1, 40, 5000])
def test_as_many_groups_as_there_may_be(m):
    groups, rows, cols = B.MWU_MAX_GROUPS, 40, 72
    gen = gen_of(m)
    which = torch.sort(torch.randint(groups, (m,), generator=gen, device="cuda"))[0]
    off = torch.searchsorted(which, torch.arange(groups + 1, device="cuda")).to(torch.int32)
    W, X, dY = normal(gen, groups, rows, cols, std=0.1), normal(gen, m, cols), normal(gen, m, rows)
    Y, dX, st = torch.empty(m, rows, device="cuda"), torch.empty(m, cols, device="cuda"), new_status()
    dW = torch.empty(groups, rows, cols, device="cuda")
    B.mwu_gemm_grouped(groups, rows, cols, W, cols, rows * cols, off, X, m, cols, Y, rows, 1, st)
    B.mwu_gemm_grouped_dx(groups, rows, cols, W, cols, rows * cols, off, dY, m, rows, dX, cols, 1, st)
    B.mwu_gemm_grouped_dw(groups, rows, cols, off, dY, m, rows, X, cols, dW, cols, rows * cols, 1, 0, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    w, x, d = W[which].to(F64), X.to(F64), dY.to(F64)
    check(Y, torch.einsum("mk,mnk->mn", x, w), torch.einsum("mk,mnk->mn", x.abs(), w.abs()), cols, 1)
    check(dX, torch.einsum("mn,mnk->mk", d, w), torch.einsum("mn,mnk->mk", d.abs(), w.abs()), rows, 1)
    one = torch.einsum("mn,mk->mnk", d, x)
    ref = torch.zeros(groups, rows, cols, dtype=F64, device="cuda").index_add_(0, which, one)
    mag = torch.zeros(groups, rows, cols, dtype=F64, device="cuda").index_add_(0, which, one.abs())
    check(dW, ref, mag, 64, 1)


@pytest.mark.parametrize("at", [[0, 5, 4, 9], [-1, 3, 5, 9], [0, 3, 5, 11], [7, 3, 5, 9], [0, 1, 2, 2 ** 31 - 1], [0, -2 ** 31, 2, 3]])
def test_offsets_that_make_no_sense_write_nothing(at):
    gen, rows, cols, m = gen_of(1), 24, 40, 10
    off = torch.tensor(at, dtype=torch.int32, device="cuda")
    W, X, dY = normal(gen, 3, rows, cols), normal(gen, m, cols), normal(gen, m, rows)
    Y, dX, dW = sentinel(m, rows, torch.float32), sentinel(m, cols, torch.float32), sentinel(3 * rows, cols, torch.float32)
    for call in (lambda st: B.mwu_gemm_grouped(3, rows, cols, W, cols, rows * cols, off, X, m, cols, Y, rows, 1, st),
                 lambda st: B.mwu_gemm_grouped_dx(3, rows, cols, W, cols, rows * cols, off, dY, m, rows, dX, cols, 1, st),
                 lambda st: B.mwu_gemm_grouped_dw(3, rows, cols, off, dY, m, rows, X, cols, dW, cols, rows * cols, 1, 0, st)):
        st = new_status()
        call(st)
        torch.cuda.synchronize()
        assert int(st.item()) == B.MWU_DEV_BOUNDS
    assert bool((Y == 777).all() & (dX == 777).all() & (dW == 777).all())


def test_the_binding_refuses_other_types_and_places():
    gen, st = gen_of(1), new_status()
    W, X, Y, off = normal(gen, 2, 24, 40), normal(gen, 9, 40), torch.zeros(9, 24, device="cuda"), torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    good = dict(groups=2, rows=24, cols=40, Wd=W, ldw=40, w_stride=960, offsets=off, X=X, M=9, ldx=40, Y=Y, ldy=24, y_dtype=1, dev_status=st)
    for change in (dict(offsets=off.long()), dict(Wd=W.float()), dict(X=X.half()), dict(y_dtype=0), dict(Y=Y.t()), dict(X=X.cpu()), dict(dev_status=st.float())):
        with pytest.raises(ValueError):
            B.mwu_gemm_grouped(**{**good, **change})
    with pytest.raises(B.MwuError):
        B.mwu_gemm_grouped(**{**good, "ldw": 36})
    B.mwu_gemm_grouped(**good)
    torch.cuda.synchronize()
    assert int(st.item()) == 0


def test_no_rows():
    gen, rows, cols = gen_of(2), 24, 40
    off, st = torch.zeros(3, dtype=torch.int32, device="cuda"), new_status()
    W, none = normal(gen, 2, rows, cols), normal(gen, 1, 40)
    Y, dW = sentinel(4, 40, torch.float32), sentinel(2 * rows, cols, torch.float32)
    B.mwu_gemm_grouped(2, rows, cols, W, cols, rows * cols, off, none, 0, cols, Y, 40, 1, st)
    B.mwu_gemm_grouped_dx(2, rows, cols, W, cols, rows * cols, off, none, 0, 40, Y, 40, 1, st)
    B.mwu_gemm_grouped_dw(2, rows, cols, off, none, 0, 40, none, 40, dW, cols, rows * cols, 1, 0, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and bool((Y == 777).all()) and bool((dW == 0).all())


def a_step(gen, groups, m, rows, cols):
    which = torch.sort(torch.randint(groups, (m,), generator=gen, device="cuda"))[0]
    off = torch.searchsorted(which, torch.arange(groups + 1, device="cuda")).to(torch.int32)
    return dict(g=groups, m=m, n=rows, k=cols, off=off, W=normal(gen, groups, rows, cols, std=0.1), X=normal(gen, m, cols),
                dY=normal(gen, m, rows), Y=torch.zeros(m, rows, device="cuda"), dX=torch.zeros(m, cols, device="cuda"),
                dW=torch.zeros(groups, rows, cols, device="cuda"), st=new_status())


def run_step(s, stream=None):
    n, k = s["n"], s["k"]
    B.mwu_gemm_grouped(s["g"], n, k, s["W"], k, n * k, s["off"], s["X"], s["m"], k, s["Y"], n, 1, s["st"], stream)
    B.mwu_gemm_grouped_dx(s["g"], n, k, s["W"], k, n * k, s["off"], s["dY"], s["m"], n, s["dX"], k, 1, s["st"], stream)
    B.mwu_gemm_grouped_dw(s["g"], n, k, s["off"], s["dY"], s["m"], n, s["X"], k, s["dW"], k, n * k, 1, 0, s["st"], stream)


def outputs(s):
    return [s[k].clone() for k in ("Y", "dX", "dW")]


def test_the_same_bits_again_on_two_streams_and_in_a_graph():
    gen = gen_of(9)
    a, b = a_step(gen, 6, 700, 264, 328), a_step(gen, 3, 1100, 520, 136)
    run_step(a)
    run_step(b)
    torch.cuda.synchronize()
    want = [outputs(a), outputs(b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, st in zip((a, b), streams):
            run_step(s, st)
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        assert int(s["st"].item()) == 0 and all(torch.equal(x, y) for x, y in zip(outputs(s), w))
    graphs = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run_step(s)
        graphs.append(g)
    # other offsets in the same buffers: the graph reads them on the device
    a["off"][1:-1] = torch.sort(torch.randint(0, a["m"] + 1, (5,), generator=gen, device="cuda"))[0].to(torch.int32)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    got = outputs(a)
    assert all(torch.equal(x, y) for x, y in zip(outputs(b), want[1]))
    run_step(a)
    torch.cuda.synchronize()
    assert int(a["st"].item()) == 0 and all(torch.equal(x, y) for x, y in zip(outputs(a), got))


def test_fp32_sums_of_long_reductions():
    """Pieces of 512 products: below 1e-6 of the result in norm, as the header says."""
    gen, m, rows, cols = gen_of(3), 8192, 256, 256
    off = torch.tensor([0, m], dtype=torch.int32, device="cuda")
    dY, X, dW, st = normal(gen, m, rows), normal(gen, m, cols), torch.empty(rows, cols, device="cuda"), new_status()
    B.mwu_gemm_grouped_dw(1, rows, cols, off, dY, m, rows, X, cols, dW, cols, rows * cols, 1, 0, st)
    ref = dY.to(F64).t() @ X.to(F64)
    assert float((dW.to(F64) - ref).norm() / ref.norm()) < 1e-6
    W, Xl = normal(gen, 1, rows, m), normal(gen, 64, m)
    Y, off = torch.empty(64, rows, device="cuda"), torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    B.mwu_gemm_grouped(1, rows, m, W, m, rows * m, off, Xl, 64, m, Y, rows, 1, st)
    ref = Xl.to(F64) @ W[0].to(F64).t()
    assert float((Y.to(F64) - ref).norm() / ref.norm()) < 1e-6


def test_bf16_sums_of_very_long_reductions():
    """More rows than go into one piece of a bf16 sum (262144), by whole numbers whose sums a bf16 result holds exactly."""
    m, rows, cols = 600011, 8, 16
    gen = gen_of(12)
    which = torch.randint(0, m, (40,), generator=gen, device="cuda")
    d, x = torch.zeros(m, rows, dtype=torch.bfloat16, device="cuda"), torch.zeros(m, cols, dtype=torch.bfloat16, device="cuda")
    d[which] = torch.randint(-2, 3, (40, rows), generator=gen, device="cuda").to(torch.bfloat16)
    x[which] = torch.randint(-1, 2, (40, cols), generator=gen, device="cuda").to(torch.bfloat16)
    off, st = torch.tensor([0, 11, 600000], dtype=torch.int32, device="cuda"), new_status()
    dW = torch.zeros(2, rows, cols, dtype=torch.bfloat16, device="cuda")
    B.mwu_gemm_grouped_dw(2, rows, cols, off, d, m, rows, x, cols, dW, cols, rows * cols, 0, 0, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for g, r in enumerate((slice(0, 11), slice(11, 600000))):
        assert torch.equal(dW[g].to(F64), d[r].to(F64).t() @ x[r].to(F64))      # below 256 in magnitude: 40 products of at most 2


def test_positions_beyond_32_bits():
    gen, rows, cols = gen_of(4), 64, 64
    m, ld = 70000, 32768                                    # the last rows start past 2^31 elements
    X = torch.zeros(m, ld, dtype=torch.bfloat16, device="cuda")
    X[:, :cols] = normal(gen, m, cols)
    stride = 3 << 29                                        # the second and third weight start past 2^31 bytes and elements
    W = torch.zeros(2 * stride + rows * cols, dtype=torch.bfloat16, device="cuda")
    for g in range(3):
        W[g * stride:g * stride + rows * cols] = normal(gen, rows * cols, std=0.1)
    at = [0, 100, m - 300, m]
    off, st = torch.tensor(at, dtype=torch.int32, device="cuda"), new_status()
    Y = torch.full((m, ld), 777.0, dtype=torch.bfloat16, device="cuda")
    B.mwu_gemm_grouped(3, rows, cols, W, cols, stride, off, X, m, ld, Y, ld, 0, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and bool((Y[-300:, rows:] == 777).all())
    for g in range(3):
        x = X[at[g]:at[g + 1], :cols].to(F64)
        w = W[g * stride:g * stride + rows * cols].view(rows, cols).to(F64).t()
        check(Y[at[g]:at[g + 1], :rows], x @ w, x.abs() @ w.abs(), cols, 0)
    del X, Y, W
    dW = torch.full((2 * stride + rows * cols,), 777.0, dtype=torch.float32, device="cuda")
    d, x = normal(gen, 500, rows), normal(gen, 500, cols)
    at = [0, 130, 177, 500]
    B.mwu_gemm_grouped_dw(3, rows, cols, torch.tensor(at, dtype=torch.int32, device="cuda"), d, 500, rows, x, cols, dW, cols, stride, 1, 0, st)
    torch.cuda.synchronize()
    for g in range(3):
        a, b = d[at[g]:at[g + 1]].to(F64).t(), x[at[g]:at[g + 1]].to(F64)
        check(dW[g * stride:g * stride + rows * cols].view(rows, cols), a @ b, a.abs() @ b.abs(), at[g + 1] - at[g], 1)
        assert float(dW[g * stride + rows * cols]) == 777.0 if g < 2 else True


def test_gradients_against_differences():
    """<dL/dW, E> and <dL/dX, E> with L = <R, Y>: Y is linear in both, so a central difference is exact but for its roundings."""
    gen, lengths, rows, cols = gen_of(6), [9, 0, 33, 22], 48, 56
    at = offsets_of(lengths)
    m, off, st = at[-1], torch.tensor(at, dtype=torch.int32, device="cuda"), new_status()
    pow2 = lambda *s: (torch.randint(-2, 3, s, generator=gen, device="cuda")).to(torch.bfloat16)      # small whole numbers: exact
    W, X, R = pow2(4, rows, cols), pow2(m, cols), pow2(m, rows)
    EW, EX = pow2(4, rows, cols), pow2(m, cols)

    def loss(w, x):
        y = torch.zeros(m, rows, device="cuda")
        B.mwu_gemm_grouped(4, rows, cols, w, cols, rows * cols, off, x, m, cols, y, rows, 1, st)
        return float((y.to(F64) * R.to(F64)).sum())

    dX, dW = torch.zeros(m, cols, device="cuda"), torch.zeros(4, rows, cols, device="cuda")
    B.mwu_gemm_grouped_dx(4, rows, cols, W, cols, rows * cols, off, R, m, rows, dX, cols, 1, st)
    B.mwu_gemm_grouped_dw(4, rows, cols, off, R, m, rows, X, cols, dW, cols, rows * cols, 1, 0, st)
    # whole numbers below 2^24 throughout: equality
    assert float((dW.to(F64) * EW.to(F64)).sum()) == (loss(W + EW, X) - loss(W - EW, X)) / 2
    assert float((dX.to(F64) * EX.to(F64)).sum()) == (loss(W, X + EX) - loss(W, X - EX)) / 2


def test_experts_compressed_then_multiplied():
    """As a layer of experts is used: every expert projected, packed and expanded into one stack, rows multiplied, gradients taken."""
    gen, groups, rows, cols, m = gen_of(8), 4, 200, 192, 333
    pad = 256                                               # mwu_decode writes whole tiles of 128 rows
    stack = torch.zeros(groups, pad, cols, dtype=torch.bfloat16, device="cuda")
    for g in range(groups):
        w = torch.randn(rows, cols, generator=gen, device="cuda") * 0.02
        blocks = rows * cols // 8
        desc = B.make_desc(rows, cols, 8, blocks // 2, blocks // 4)
        bufs = B.ProjectionBuffers(desc)
        bufs.project(w)
        packed = bufs.pack(w)
        B.mwu_decode(desc, packed, stack[g], cols, bufs.dev_status)
        x1 = normal(gen, 5, cols)
        y1, y2 = torch.empty(5, rows, device="cuda"), torch.empty(5, rows, device="cuda")
        B.mwu_gemm(desc, packed, x1, 5, cols, y1, rows, 1, bufs.dev_status)
        B.mwu_gemm_grouped(1, rows, cols, stack[g], cols, pad * cols, torch.tensor([0, 5], dtype=torch.int32, device="cuda"), x1, 5,
                           cols, y2, rows, 1, bufs.dev_status)
        torch.cuda.synchronize()
        assert int(bufs.dev_status.item()) == 0
        mag = x1.to(F64).abs() @ stack[g, :rows].to(F64).abs().t()
        assert bool(((y1.to(F64) - y2.to(F64)).abs() <= 2 * (cols / 8 + 8) * 2.0 ** -23 * mag).all())
    s = a_step(gen, groups, m, rows, cols)
    B.mwu_gemm_grouped(groups, rows, cols, stack, cols, pad * cols, s["off"], s["X"], m, cols, s["Y"], rows, 1, s["st"])
    B.mwu_gemm_grouped_dx(groups, rows, cols, stack, cols, pad * cols, s["off"], s["dY"], m, rows, s["dX"], cols, 1, s["st"])
    torch.cuda.synchronize()
    at = s["off"].tolist()
    for g in range(groups):
        r, w = slice(at[g], at[g + 1]), stack[g, :rows].to(F64)
        x, d = s["X"][r].to(F64), s["dY"][r].to(F64)
        check(s["Y"][r], x @ w.t(), x.abs() @ w.t().abs(), cols, 1)
        check(s["dX"][r], d @ w, d.abs() @ w.abs(), rows, 1)
