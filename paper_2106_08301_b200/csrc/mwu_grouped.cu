// Grouped products: rows sorted by group, one weight per group, lengths that only the device knows.
//
//   mwu_gemm_grouped      Y[m]  = X[m] . W_g^T     reduction over cols
//   mwu_gemm_grouped_dx   dX[m] = dY[m] . W_g      reduction over rows (of the weights)
//   mwu_gemm_grouped_dw   dW_g  = dY_g^T . X_g     reduction over the rows of the group
//
// One kernel serves all three.  A cluster of two CTAs computes tiles of 256 "features" by up to 256 "lines" with
// tcgen05.mma.cta_group::2, where features are the contiguous axis of the output and lines its rows:
//
//   product        features = weight rows,    lines = activation rows,  operands K-major, K-major
//   input grad     features = weight columns, lines = gradient rows,    operands MN-major (W as it lies), K-major
//   weight grad    features = weight columns, lines = weight rows,      operands MN-major (X), MN-major (dY)
//
// The weights are the M side of the instruction, so a group of few rows costs an N of 32 instead of a half empty tile of 128,
// and a lane of tensor memory is a feature, so a warp's store of one line is one contiguous run of the output, whatever
// the line: ragged groups need no masked box, only a test per line.
// The groups' offsets are checked and turned into a table of tiles by every CTA at its start (device memory, no host).
// In the weight gradient a group's last block of 64 rows may hold rows of the next group, which must not be multiplied, not
// even by zero (they may be NaN): its stage is loaded onto a barrier of its own, a warp of each CTA zeroes the
// foreign rows up to the next multiple of 16 in both operands, and only then it is handed to the issuer of the MMAs.
// fp32 results: the tensor core drops what lies below an accumulator's last place (about 1e-9 of the result a product, always
// towards zero), so sums are taken out of tensor memory every 512 products and added in registers; bf16 results hide it.
//
// What bounds it (us a pass among others, 3 % either way from one device to the next).  Many rows: loads, and tiles dealt to the pairs
// in a fixed order.  16 of 4096 x 4096, 16384 rows: 465, 1.18 PFLOP/s (300 to 357 without the loads); input gradient of 8192 rows 268, alone
// and cool 217 with the tensor pipe at 70 % and the crossbar at 41 %.  At 0.37 us for 256 x 256 x 64 products the busiest pair has 364 of
// the product's time where the mean is 331, 186 and 170 of the input gradient's, 184 and 169 of the weight gradient's; MN-major operands come
// in boxes of half a width; one lane issues the MMAs of all tiles; and passes in a row run into the power cap (1.55 GHz).  Weight
// gradients: the fp32 output besides (16 of 2048 x 4096: 327, 253 without the stores; a burst of them from all SMs leaves at 5.8 TB/s).  Few rows: reading the weights (64 of 2048 x 4096, 256 rows: 166, 5.9 TB/s).  Small calls: 2.5 us until the
// roles begin, 2.3 until the first stage is there, 2 to 3 from the last MMA to the last store, and 0.27 us a stage whatever is in it.
// Tried and taken back: weights or activations brought to L2 ahead of their loads (4 to 17 % slower: the copy engine's requests are what
// is short); tiles of a pair worked out in a table before the first load, and the epilogue's code in one loop (a small call 1.3 us
// slower); six stages with one output box a warp, and three boxes (no change); letting the kernel behind start early (2 rows 8.65 instead of 8.98,
// but five calls in a row, rank 64, 134.5 instead of 128.6).
//
// Roles per CTA (11 warps): warp 0 TMA producer, warp 1 tensor memory and (leader) MMAs, warps 2 to 9 epilogue (two per
// 32-lane quarter, every other 32 lines), warp 10 zeroes foreign rows.  Every wait on an mbarrier is bounded; when one runs
// out the kernel raises MWU_DEV_TIMEOUT, lets its loads land, frees tensor memory and returns.
#include "mwu_rows.cuh"

namespace mwu {
namespace gemm {

EncodeTiledFn get_encode_fn();          // mwu_gemm.cu

constexpr int G_RING = 180 * 1024;                   // bytes of stages
constexpr int G_MOST_STAGES = 16;
constexpr int G_EPI_WARPS = 8;
constexpr int G_FIX_WARP = 2 + G_EPI_WARPS;
constexpr int G_THREADS = 32 * (3 + G_EPI_WARPS);
constexpr int G_SIDE = 128 * 128;                    // bytes of 128 features or lines x 64 reduction steps
constexpr int G_SUB = 64 * 128;                      // MN-major: 64 features x 64 reduction steps
constexpr int G_BOX = 2048;                          // of output: 32 features x 16 lines of fp32, x 32 of bf16; two to a warp
constexpr int G_BAND = 8;                            // line tiles per band of the tile order
constexpr int G_CHUNK = 8;                           // blocks of 64 between two sums of an fp32 result (512 products)
constexpr int G_CHUNK_BF16 = 4096;                   // ... of a bf16 result: 262144 products lose 3e-4 of it and take 1 ms

enum { G_FORWARD = 0, G_DX = 1, G_DW = 2 };

struct GroupedParams {
    const int *offsets;                 // [groups + 1]
    void *out;
    long long ldo, out_stride;          // elements between output rows, between groups (weight gradient)
    int groups, M;
    int features, reduction, lines;     // reduction: of a product or input gradient; lines: of a weight gradient
    int line_tile;                      // most lines of a tile (a multiple of 32)
    int feature_box;                    // product: weight rows of a box, as many as a CTA has of few features
    int feature_side, block_bytes;      // of 64 reduction steps: bytes of features, of all
    int blocks, stages;                 // blocks of a stage, stages of the ring
    int out_fp32, accumulate;
    WaitLimits wait;
    unsigned *dev_status;
};

// The lines of a CTA's half tile as few boxes, whose issue takes as long as some of their transfer: 128 lines (from 97 on; what is
// too many is never multiplied), 64 and 32, 64, or 32.  A weight gradient's boxes are 64 lines wide by 64 rows and take only m[0].
struct LineMaps { CUtensorMap m[3]; };
__host__ __device__ __forceinline__ int boxed_lines(int half) { return half > 96 ? 128 : (half + 31) & ~31; }

struct GroupedSmem {
    unsigned long long full[G_MOST_STAGES], empty[G_MOST_STAGES], tail[G_MOST_STAGES], peer_fixed[G_MOST_STAGES], tfull[2], tempty[2], drain;
    unsigned tmem_base;
    int abort, drain_abort;
    int n_live;                         // groups with rows
    int offsets[MWU_MAX_GROUPS + 1];
    int cum[MWU_MAX_GROUPS + 1];        // line tiles before the i-th group with rows
    unsigned short live[MWU_MAX_GROUPS];
};

static_assert(1024 + G_RING + G_EPI_WARPS * 2 * G_BOX + sizeof(GroupedSmem) <= 232448, "grouped kernel: shared memory above 227 KB");

__device__ __forceinline__ void tma_load_3d_pair(unsigned dst, const CUtensorMap *map, unsigned bar_cluster, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 "
        "[%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar_cluster), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, unsigned src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap *map, unsigned src, int x, int y, int z) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
// MN-major operand, 128-byte swizzle: 64 features to a row of 128 bytes, 8 reduction steps to 1024 bytes, the next 64 features
// G_SUB bytes on
__device__ __forceinline__ unsigned long long make_desc_mn(unsigned smem_addr) {
    unsigned long long d = 0;
    d |= (unsigned long long)((smem_addr & 0x3FFFFu) >> 4);
    d |= (unsigned long long)(G_SUB >> 4) << 16;
    d |= (unsigned long long)(1024 >> 4) << 32;
    d |= (unsigned long long)1 << 46;
    d |= (unsigned long long)2 << 61;
    return d;
}
// a wait that also orders what another CTA of the cluster wrote before it arrived
__device__ __forceinline__ bool mbar_wait_cluster(unsigned bar, unsigned parity, volatile int *abort, long long limit) {
    const long long t0 = clock64();
#pragma unroll 1
    while (true) {
        unsigned ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if (*abort) return false;
        if (clock64() - t0 > limit) { *abort = 1; return false; }
    }
}

// Bytes of features that the CTA with features f0 .. f0 + 127 of a tile loads for a stage: what lies wholly behind the last feature is
// left out, since a lane without a feature may hold anything (a side as long as an adapter's rank: a quarter of the loads).
template <int OP>
__device__ __forceinline__ unsigned feature_bytes(const GroupedParams &p, int f0) {
    if (f0 >= p.features) return 0u;
    return OP == G_FORWARD ? (unsigned)p.feature_box * 128u : (f0 + 64 < p.features ? 2u : 1u) * (unsigned)G_SUB;
}

struct GroupedTile {
    int group, feature0, line0, line_count, line_pad;   // line0: row of X / dY, or weight row
    int red0, red_len;                                  // weight gradient: first row of the group and their number
};

// Tile t.  Tiles of a group lie together; inside it they walk bands of G_BAND line tiles, feature tile by feature tile, so
// that the pairs running at one time share a few tiles of either operand in L2.
template <int OP>
__device__ __forceinline__ void grouped_tile(const GroupedParams &p, const GroupedSmem *sm, unsigned t, unsigned f_tiles, GroupedTile &o) {
    unsigned lt, n_lt, r;
    if (OP == G_DW) {
        n_lt = (unsigned)(p.lines + p.line_tile - 1) / (unsigned)p.line_tile;
        const unsigned per = n_lt * f_tiles, g = t / per;
        r = t - g * per;
        o.group = (int)g;
        o.red0 = sm->offsets[g];
        o.red_len = sm->offsets[g + 1] - o.red0;
    } else {
        const unsigned q = t / f_tiles;                     // the line tile that would be it if a group's were the outer loop
        int lo = 0, hi = sm->n_live - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((unsigned)sm->cum[mid] <= q) lo = mid; else hi = mid - 1;
        }
        o.group = sm->live[lo];
        n_lt = (unsigned)(sm->cum[lo + 1] - sm->cum[lo]);
        r = t - (unsigned)sm->cum[lo] * f_tiles;
    }
    const unsigned per_band = G_BAND * f_tiles, band = r / per_band, rb = r - band * per_band;
    const unsigned left = n_lt - band * G_BAND, wide = left < (unsigned)G_BAND ? left : (unsigned)G_BAND;
    const unsigned ft = rb / wide;
    lt = band * G_BAND + (rb - ft * wide);
    o.feature0 = (int)(ft * 256);
    if (OP == G_DW) {
        o.line0 = (int)lt * p.line_tile;
        o.line_count = min(p.line_tile, p.lines - o.line0);
    } else {
        const int begin = sm->offsets[o.group], len = sm->offsets[o.group + 1] - begin;
        // as many lines to every tile of the group, in whole 32s: never more than line_tile, and no tile is left empty
        const int h = (((len + (int)n_lt - 1) / (int)n_lt) + 31) & ~31;
        o.line0 = begin + (int)lt * h;
        o.line_count = min(h, len - (int)lt * h);
        o.red0 = 0;
        o.red_len = p.reduction;
    }
    o.line_pad = (o.line_count + 31) & ~31;
}

template <int OP, int BL>
__global__ void __launch_bounds__(G_THREADS, 1)
mwu_gemm_grouped_kernel(const __grid_constant__ CUtensorMap tmap_f, const __grid_constant__ LineMaps maps_l,
                        const __grid_constant__ CUtensorMap tmap_out, const __grid_constant__ GroupedParams p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *ring = smem_raw + smem_pad_1024(smem_raw);
    unsigned char *boxes_out = ring + G_RING;
    GroupedSmem *sm = reinterpret_cast<GroupedSmem *>(boxes_out + G_EPI_WARPS * 2 * G_BOX);
    volatile int *abort = &sm->abort;
    // (the same in all lanes, and known to be: what hangs on it then lives in uniform registers, which MMAs and copies take their operands from)
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const unsigned rank = cluster_rank();               // 0: leader (issues the MMAs), 1: peer
    const unsigned pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const unsigned f_tiles = (unsigned)(p.features + 255) / 256;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(smem_u32(&sm->full[s]), 1 + (s == p.wait.dead_slot));
            mbar_init(smem_u32(&sm->empty[s]), 1);
            mbar_init(smem_u32(&sm->tail[s]), 1 + (s == p.wait.dead_slot));
            mbar_init(smem_u32(&sm->peer_fixed[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sm->tfull[b]), 1);
            mbar_init(smem_u32(&sm->tempty[b]), 2 * G_EPI_WARPS);
        }
        mbar_init(smem_u32(&sm->drain), 1);
        sm->abort = 0;
        sm->drain_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&tmap_f);
        prefetch_map(&tmap_out);
        for (int b = 0; b < (OP == G_DW ? 1 : 3); ++b) prefetch_map(&maps_l.m[b]);
    }
    __syncwarp();
    cluster_arrive();                                   // both CTAs' barriers exist before any remote arrive: waited for below
    if (warp == 1) tmem_alloc2(smem_u32(&sm->tmem_base), 512);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // the groups: offsets in order and inside the rows that there are, or nothing is done at all
    int bad = 0;
    for (int i = threadIdx.x; i <= p.groups; i += G_THREADS) {
        const int v = __ldg(p.offsets + i), before = i ? __ldg(p.offsets + i - 1) : 0;
        sm->offsets[i] = v;
        bad |= v < before || v > p.M;
    }
    bad = __syncthreads_or(bad);
    if (bad && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.dev_status, (unsigned)MWU_DEV_BOUNDS);
    if (OP != G_DW && warp == 2) {
        int n = 0, tiles = 0;
        for (int g0 = 0; g0 < p.groups; g0 += 32) {
            const int g = g0 + lane;
            const int len = g < p.groups && !bad ? sm->offsets[g + 1] - sm->offsets[g] : 0;
            const int mine = len > 0 ? (int)(((unsigned)len + (unsigned)p.line_tile - 1) / (unsigned)p.line_tile) : 0;
            int upto = mine;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int o = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += o;
            }
            const unsigned some = __ballot_sync(0xffffffffu, mine > 0);
            if (mine) {
                const int at = n + __popc(some & ((1u << lane) - 1u));
                sm->live[at] = (unsigned short)g;
                sm->cum[at] = tiles + upto - mine;
            }
            n += __popc(some);
            tiles += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lane == 0) {
            sm->cum[n] = tiles;
            sm->n_live = n;
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_wait();
    tc_fence_after();
    const unsigned tmem_base = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile unsigned *>(&sm->tmem_base), 0);
    // (the host refuses sizes whose tile count could pass 2^31)
    const unsigned total = bad ? 0u : OP == G_DW ? (unsigned)p.groups * f_tiles * ((unsigned)(p.lines + p.line_tile - 1) / (unsigned)p.line_tile)
                                                 : (unsigned)sm->cum[sm->n_live] * f_tiles;
    GroupedTile t;

    if (warp == 0) {
        // ---------------- TMA producer: this CTA's halves of both operands ----------------
        int stage = 0;
        unsigned phase = 0, tails = 0;                     // tails: bit s set after an odd number of them in slot s
        bool ok = true;
        for (unsigned k = pair; ok && k < total; k += n_pairs) {
            grouped_tile<OP>(p, sm, k, f_tiles, t);
            const int n_blk = (t.red_len + 63) / 64, half = t.line_pad / 2;
            const int f0 = t.feature0 + (int)rank * 128, l0 = t.line0 + (int)rank * half;
            const int boxes = (half + 63) / 64, boxed = boxed_lines(half);
            const unsigned line_bytes = OP == G_DW ? (unsigned)boxes * G_SUB : (unsigned)boxed * 128u;
            const unsigned mine = feature_bytes<OP>(p, f0), pair_bytes = feature_bytes<OP>(p, t.feature0) + feature_bytes<OP>(p, t.feature0 + 128) + 2 * line_bytes;
            for (int b0 = 0; b0 < n_blk; b0 += BL) {
                ok = warp_wait_spin(smem_u32(&sm->empty[stage]), phase ^ 1u, abort, p.wait.cycles);
                if (!ok) break;
                const int nb = min(BL, n_blk - b0), last = t.red_len - (b0 + nb - 1) * 64;     // reduction steps from the last block on
                const bool tail = OP == G_DW && last < 64 && (last & 15);
                if (elect_one()) {
                    unsigned df = smem_u32(ring) + (unsigned)(stage * BL * p.block_bytes);
                    if (tail) {
                        // foreign rows to zero: onto this CTA's own barrier, the fixing warp hands the stage on.  (A barrier to a
                        // slot: the next group's last stage may be under way before this one has landed.)
                        const unsigned bar = smem_u32(&sm->tail[stage]);
                        mbar_expect_tx(bar, (unsigned)nb * (mine + line_bytes));
                        for (int b = 0; b < nb; ++b, df += (unsigned)p.block_bytes) {
                            const unsigned dl = df + (unsigned)p.feature_side;
                            const int row = t.red0 + (b0 + b) * 64;
                            if (mine) tma_load_2d(df, &tmap_f, bar, f0, row);
                            if (mine > G_SUB) tma_load_2d(df + G_SUB, &tmap_f, bar, f0 + 64, row);
                            for (int j = 0; j < boxes; ++j) tma_load_2d(dl + j * G_SUB, &maps_l.m[0], bar, l0 + 64 * j, row);
                        }
                    } else {
                        const unsigned bar = mbar_addr_in_cta(smem_u32(&sm->full[stage]), 0);
                        if (rank == 0) mbar_expect_tx(smem_u32(&sm->full[stage]), (unsigned)nb * pair_bytes);
                        for (int b = 0; b < nb; ++b, df += (unsigned)p.block_bytes) {
                            const unsigned dl = df + (unsigned)p.feature_side;
                            const int r0 = (b0 + b) * 64;
                            if (OP == G_FORWARD) {
                                if (mine) tma_load_3d_pair(df, &tmap_f, bar, r0, f0, t.group);
                            } else if (OP == G_DX) {
                                if (mine) tma_load_3d_pair(df, &tmap_f, bar, f0, r0, t.group);
                                if (mine > G_SUB) tma_load_3d_pair(df + G_SUB, &tmap_f, bar, f0 + 64, r0, t.group);
                            } else {
                                if (mine) tma_load_2d_pair(df, &tmap_f, bar, f0, t.red0 + r0);
                                if (mine > G_SUB) tma_load_2d_pair(df + G_SUB, &tmap_f, bar, f0 + 64, t.red0 + r0);
                            }
                            if (OP == G_DW) {
                                for (int j = 0; j < boxes; ++j) tma_load_2d_pair(dl + j * G_SUB, &maps_l.m[0], bar, l0 + 64 * j, t.red0 + r0);
                            } else {
                                if (boxed == 128) tma_load_2d_pair(dl, &maps_l.m[0], bar, r0, l0);
                                else if (boxed & 64) tma_load_2d_pair(dl, &maps_l.m[1], bar, r0, l0);
                                if (boxed & 32) tma_load_2d_pair(dl + (boxed & 64) * 128, &maps_l.m[2], bar, r0, l0 + (boxed & 64));
                            }
                        }
                    }
                }
                __syncwarp();
                tails ^= (unsigned)tail << stage;
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
        // a wait ran out: the loads in flight (of both CTAs, as far as they were issued) land before anybody leaves
        if (__any_sync(0xffffffffu, *abort)) {
            volatile int *drain_abort = &sm->drain_abort;
            if (rank == 0)
                for (int s = 0; s < p.stages; ++s) mbar_wait(smem_u32(&sm->full[s]), s < stage ? phase : phase ^ 1u, drain_abort, p.wait.cycles);
            for (int s = 0; s < p.stages; ++s) mbar_wait(smem_u32(&sm->tail[s]), ((tails >> s) & 1u) ^ 1u, drain_abort, p.wait.cycles);
            __syncwarp();
        }
    } else if (warp == 1 && rank == 0) {
        // ---------------- MMA issuer (leader) ----------------
        int stage = 0;
        unsigned phase = 0, use = 0;
        bool ok = true;
        const bool leader = elect_one();                    // the lane that issues
        for (unsigned k = pair; ok && k < total; k += n_pairs) {
            grouped_tile<OP>(p, sm, k, f_tiles, t);
            const int red_len = __shfl_sync(0xffffffffu, t.red_len, 0), n_blk = (red_len + 63) / 64, chunk = p.out_fp32 ? G_CHUNK : G_CHUNK_BF16;
            const unsigned idesc = make_idesc_pair(__shfl_sync(0xffffffffu, t.line_pad, 0)) | (OP != G_FORWARD ? 1u << 15 : 0u) | (OP == G_DW ? 1u << 16 : 0u);
            for (int c0 = 0; ok && c0 < n_blk; c0 += chunk, ++use) {
                const unsigned buf = use & 1u;
                ok = warp_wait_spin(smem_u32(&sm->tempty[buf]), ((use >> 1) & 1u) ^ 1u, abort, p.wait.cycles);
                if (!ok) break;
                tc_fence_after();
                const int c1 = min(n_blk, c0 + chunk);
                for (int b0 = c0; b0 < c1; b0 += BL) {
                    // (No vote, no election and no warp barrier in this loop: where the limit runs out lanes may leave it at different
                    // stages, and the vote behind it is the first place where they need one another again.)
                    if (!mbar_wait_spin(smem_u32(&sm->full[stage]), phase, abort, p.wait.cycles)) { ok = false; break; }
                    tc_fence_after();
                    const int nb = min(BL, n_blk - b0);
                    unsigned af = smem_u32(ring) + (unsigned)(stage * BL * p.block_bytes);
                    if (leader) {
                        for (int b = b0; b < b0 + nb; ++b, af += (unsigned)p.block_bytes) {
                            const unsigned al = af + (unsigned)p.feature_side;
                            const unsigned long long fdesc = OP == G_FORWARD ? make_desc(af) : make_desc_mn(af);
                            const unsigned long long ldesc = OP == G_DW ? make_desc_mn(al) : make_desc(al);
                            const int steps = min(4, (red_len - b * 64 + 15) / 16);
#pragma unroll
                            for (int k4 = 0; k4 < 4; ++k4)
                                if (k4 < steps)             // 16 products on: 32 bytes K-major, two groups of 8 rows MN-major
                                    umma2_bf16(tmem_base + buf * 256u, fdesc + (unsigned long long)(k4 * (OP == G_FORWARD ? 2 : 128)),
                                               ldesc + (unsigned long long)(k4 * (OP == G_DW ? 128 : 2)), idesc, (b > c0 || k4) ? 1u : 0u);
                        }
                        umma2_commit_both(smem_u32(&sm->empty[stage]));
                    }
                    if (++stage == p.stages) { stage = 0; phase ^= 1u; }
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (leader) umma2_commit_both(smem_u32(&sm->tfull[buf]));
                __syncwarp();
            }
        }
        // everything this thread issued must have retired before tensor memory is freed
        if (leader) umma2_commit_local(smem_u32(&sm->drain));
        __syncwarp();
        mbar_wait(smem_u32(&sm->drain), 0, &sm->drain_abort, p.wait.cycles);
        __syncwarp();
    } else if (warp == G_FIX_WARP) {
        // ---------------- foreign rows of a group's last stage ----------------
        if (OP == G_DW) {
            unsigned pos = 0, tails = 0;                    // pos: place of the tile's first stage in the ring; tails as in the producer
            long long behind = 0;                           // stages since the last one handed on: the limit is for each of them
            bool ok = true;
            for (unsigned k = pair; ok && k < total; k += n_pairs) {
                grouped_tile<OP>(p, sm, k, f_tiles, t);
                const unsigned n_blk = (unsigned)(t.red_len + 63) / 64, n_st = (n_blk + (unsigned)BL - 1) / (unsigned)BL;
                const int rem = t.red_len & 63;
                behind += n_st;
                if (rem & 15) {
                    const unsigned stage = (pos + n_st - 1) % (unsigned)p.stages;
                    ok = warp_wait_spin(smem_u32(&sm->tail[stage]), (tails >> stage) & 1u, abort, p.wait.cycles * behind);
                    if (!ok) break;
                    behind = 0;
                    // rows rem .. of the next multiple of 16, 128 bytes each, in the sub-tiles of either operand
                    const int rows = 16 - (rem & 15);
                    unsigned char *block = ring + (stage * (unsigned)BL + (n_blk - 1) % (unsigned)BL) * (unsigned)p.block_bytes;
                    for (int i = lane; i < rows * 32; i += 32) {
                        const int r = rem + (i >> 5), at = ((i >> 3) & 3) * G_SUB, piece = i & 7;      // at: the sub-tiles lie one behind the other
                        if (at < p.block_bytes) *reinterpret_cast<uint4 *>(block + at + r * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (rank) {
                        if (lane == 0) mbar_arrive_cluster(smem_u32(&sm->peer_fixed[stage]), 0);
                    } else {
                        ok = __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&sm->peer_fixed[stage]), (tails >> stage) & 1u, abort, p.wait.cycles));
                        if (!ok) break;
                        fence_proxy_async();
                        if (lane == 0) mbar_arrive(smem_u32(&sm->full[stage]));
                    }
                    __syncwarp();
                    tails ^= 1u << stage;
                }
                pos = (pos + n_st) % (unsigned)p.stages;
            }
        }
    } else if (warp >= 2) {
        // ---------------- epilogue: this CTA's 128 features x the tile's lines ----------------
        const int quarter = warp & 3;                       // TMEM lanes this warp may read
        const int odd = (warp - 2) >> 2;                    // its share: every other 32 lines
        unsigned use = 0;
        bool ok = true;
        unsigned char *stg = boxes_out + (warp - 2) * 2 * G_BOX;
        unsigned box_at = 0;
        const unsigned box_flip = G_BOX;
        auto next_box = [&]() {                             // the other box of the two, read by the store before last
            unsigned char *box = stg + box_at;
            box_at ^= box_flip;
            if (lane == 0) bulk_wait_read_1();
            __syncwarp();
            return box;
        };
        auto send_box = [&](const unsigned char *box, int x, int y, int z) {
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                if (OP != G_DW) tma_store_2d(&tmap_out, smem_u32(box), x, y);
                else if (p.accumulate) tma_add_3d(&tmap_out, smem_u32(box), x, y, z);
                else tma_store_3d(&tmap_out, smem_u32(box), x, y, z);
                bulk_commit();
            }
        };
        for (unsigned k = pair; ok && k < total; k += n_pairs) {
            grouped_tile<OP>(p, sm, k, f_tiles, t);
            const int n_st = (t.red_len + 63) / 64, chunk = p.out_fp32 ? G_CHUNK : G_CHUNK_BF16;
            float acc[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 32; ++j) acc[q][j] = 0.f;
            for (int c0 = 0; c0 < n_st; c0 += chunk, ++use) {
                const unsigned buf = use & 1u;
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm->tfull[buf]), (use >> 1) & 1u, abort, p.wait.cycles));
                if (!ok) break;
                tc_fence_after();
                const unsigned trow = tmem_base + ((unsigned)(quarter * 32) << 16) + buf * 256u + (unsigned)(odd * 32);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (64 * q + 32 * odd < t.line_pad) {
                        unsigned v[32];
                        tmem_ld32(trow + (unsigned)(64 * q), v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[q][j] += __uint_as_float(v[j]);
                    }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (rank == 0) mbar_arrive(smem_u32(&sm->tempty[buf]));
                    else mbar_arrive_cluster(smem_u32(&sm->tempty[buf]), 0);
                }
            }
            if (!ok) break;
            const int f0 = t.feature0 + (int)rank * 128 + quarter * 32, f = f0 + lane;
            // Output through boxes in shared memory and TMA, 40 GB/s an SM (plain stores 14 a word a lane, 21 at 16 bytes), where it is whole
            // boxes: the map clips a store at 16 bytes, and at the last weight row, but not at the end of a group of lines.
            const bool boxed = f0 + 32 <= p.features || p.features % (p.out_fp32 ? 4 : 8) == 0;
            // (accumulating: a group without rows adds nothing)
            const int lines = f0 >= p.features || (OP == G_DW && p.accumulate && n_st == 0) ? 0 : t.line_count;
            const long long row0 = (OP == G_DW ? t.group * p.out_stride : 0ll) + (long long)t.line0 * p.ldo + f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int l0 = 64 * q + 32 * odd;
                if (l0 >= lines) break;
                const int n = min(32, lines - l0);
                if (boxed && (OP == G_DW || n == 32)) {
                    if (p.out_fp32) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (OP == G_DW && 16 * h >= n) break;
                            float *box = reinterpret_cast<float *>(next_box());
#pragma unroll
                            for (int j = 0; j < 16; ++j) box[j * 32 + lane] = acc[q][16 * h + j];
                            send_box(reinterpret_cast<unsigned char *>(box), f0, t.line0 + l0 + 16 * h, t.group);
                        }
                    } else {
                        __nv_bfloat16 *box = reinterpret_cast<__nv_bfloat16 *>(next_box());
#pragma unroll
                        for (int j = 0; j < 32; ++j) box[j * 32 + lane] = __float2bfloat16_rn(acc[q][j]);
                        send_box(reinterpret_cast<unsigned char *>(box), f0, t.line0 + l0, t.group);
                    }
                } else if (f < p.features) {
                    if (p.out_fp32) {
                        float *dst = reinterpret_cast<float *>(p.out) + row0 + l0 * p.ldo;
                        if (OP == G_DW && p.accumulate) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < n) acc[q][j] += dst[j * p.ldo];
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (j < n) dst[j * p.ldo] = acc[q][j];
                    } else {
                        __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + row0 + l0 * p.ldo;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (j < n) dst[j * p.ldo] = __float2bfloat16_rn(acc[q][j]);
                    }
                }
                __syncwarp();
            }
        }
        if (lane == 0) bulk_wait_all();                     // this warp's stores are done
        __syncwarp();
    }

    // teardown: nobody leaves while the other CTA may still read this one's memory or barriers
    tc_fence_before();
    __syncthreads();
    if (*abort && threadIdx.x == 0) atomicOr(p.dev_status, (unsigned)MWU_DEV_TIMEOUT);
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc2(tmem_base, 512);
    }
}

// testing aid (see mwu.h)
static std::atomic<long long> g_rows_limit{WAIT_LIMIT_CYCLES};
static std::atomic<int> g_rows_dead_slot{-1};
WaitLimits wait_limits() { return {g_rows_limit.load(std::memory_order_relaxed), g_rows_dead_slot.load(std::memory_order_relaxed)}; }
static void set_wait_limits(long long cycles, long long slot) {
    g_rows_limit.store(cycles > 0 ? cycles : WAIT_LIMIT_CYCLES, std::memory_order_relaxed);
    g_rows_dead_slot.store(slot >= 0 && slot < G_MOST_STAGES ? (int)slot : -1, std::memory_order_relaxed);
}

template <int OP, int BL>
static cudaError_t launch_grouped_bl(const CUtensorMap &tmap_f, const LineMaps &maps_l, const CUtensorMap &tmap_out, const GroupedParams &p, long long most_tiles,
                                  int sm_count, cudaStream_t st) {
    auto kern = mwu_gemm_grouped_kernel<OP, BL>;
    const size_t smem = 1024 + (size_t)G_RING + (size_t)G_EPI_WARPS * 2 * G_BOX + sizeof(GroupedSmem);
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const long long pairs = most_tiles < sm_count / 2 ? most_tiles : sm_count / 2;
    count_launch();
    return launch_chained(kern, dim3((unsigned)(2 * pairs)), dim3(G_THREADS), smem, st, 2, tmap_f, maps_l, tmap_out, p);
}

template <int OP>
static cudaError_t launch_grouped(const CUtensorMap &tmap_f, const LineMaps &maps_l, const CUtensorMap &tmap_out, const GroupedParams &p,
                                  long long most_tiles, int sm_count, cudaStream_t st) {
    if constexpr (OP != G_DW)
        if (p.blocks == 2) return launch_grouped_bl<OP, 2>(tmap_f, maps_l, tmap_out, p, most_tiles, sm_count, st);
    return launch_grouped_bl<OP, 1>(tmap_f, maps_l, tmap_out, p, most_tiles, sm_count, st);
}

// box of 64 elements of the contiguous axis by `box_rows`, one group
static bool encode_bf16(EncodeTiledFn encode, CUtensorMap *tm, const void *ptr, int64_t inner, int64_t rows, int64_t ld, int box_rows,
                        int64_t groups, int64_t stride) {
    const cuuint64_t gdim[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)groups};
    const cuuint64_t gstride[2] = {(cuuint64_t)ld * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {(cuuint32_t)BK, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, groups ? 3 : 2, const_cast<void *>(ptr), gdim, gstride, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// an output box: 32 features of 16 lines of fp32, of 32 of bf16
static bool encode_out(EncodeTiledFn encode, CUtensorMap *tm, void *ptr, bool fp32, int64_t features, int64_t lines, int64_t ld,
                       int64_t groups, int64_t stride) {
    const int64_t size = fp32 ? 4 : 2;
    const cuuint64_t gdim[3] = {(cuuint64_t)features, (cuuint64_t)lines, (cuuint64_t)groups};
    const cuuint64_t gstride[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(stride * size)};
    const cuuint32_t box[3] = {32, (cuuint32_t)(fp32 ? 16 : 32), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return encode(tm, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, groups ? 3 : 2, ptr, gdim, gstride, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Most lines of a tile: what makes the shares of the CTA pairs take least, by an estimate in microseconds of a stage (its loads, which
// the tensor cores wait for: 0.2 for 128 features and for 128 lines each) and of a tile's output.  `lines` in runs of which there are
// `runs`, of unknown length: half a tile of each is taken to be lost.  (8192 rows of 4 groups, 4096 -> 64: 27 us with 128 lines, 31 with 256,
// both with five stages; 256 rows of 64 groups, 4096 -> 2048: 170 with 64, whose ring is longer, 179 with 256.)
static int choose_line_tile(double lines, double runs, double copies, int64_t features, double stages, double out_us, int pairs) {
    const double f_tiles = (double)((features + 255) / 256), per_feature = features >= 256 ? 0.2 : 0.2 * (double)((features + 63) / 64) / 4;
    if (lines <= 24 * runs) return 64;                      // hardly a group has more: small stages, a long ring
    double best = 1e30;
    int tile = 256;
    const int sizes[4] = {256, 192, 128, 64};
    for (int t : sizes) {
        const double tiles = f_tiles * copies * (lines / t + 0.5 * runs), rounds = tiles <= pairs ? 1.0 : tiles / pairs + 0.5;
        const double us = rounds * (0.8 + stages * (0.05 + per_feature + 0.2 * t / 256) + out_us * t / 256);
        if (us < 0.97 * best) { best = us; tile = t; }
    }
    return tile;
}

// Stages of what a CTA's share of the widest tile takes, as many as fit: loads are 2 us on their way.  A stage costs 0.27 us whatever
// it holds (the commits that hand its slot back to both CTAs follow one another at that pace), so small blocks go two to a stage
// (8192 rows 4096 -> 64: 23.5 us, 26 with one; 2 rows of 1024 x 1024: 9.2, 10.0), but not where three stages would be left (weight
// gradients of a side of 64: 28.7, 25.6 with one), and in a kernel of its own (full tiles: 2 to 6 % slower with the loop).
static void lay_out_ring(GroupedParams &p, int feature_side, int line_side, bool pairs) {
    p.feature_side = feature_side;
    p.block_bytes = feature_side + line_side;
    p.blocks = pairs && p.block_bytes <= 20 * 1024 ? 2 : 1;
    const int fit = G_RING / (p.blocks * p.block_bytes);
    p.stages = fit < G_MOST_STAGES ? fit : G_MOST_STAGES;
}

// Y = X . W^T and dX = dY . W: `red` / `features` = cols / rows of the weights, or rows / cols
template <int OP>
static int run_lines(int64_t groups, int64_t rows, int64_t cols, const void *Wd, int64_t ldw, int64_t w_stride, const int32_t *offsets,
                     const void *in, int64_t M, int64_t ldi, void *out, int64_t ldo, int32_t out_dtype, uint32_t *dev_status,
                     void *cuda_stream) {
    const int64_t features = OP == G_FORWARD ? rows : cols, red = OP == G_FORWARD ? cols : rows;
    if (!Wd || !offsets || !dev_status || M < 0 || (M > 0 && (!in || !out))) return MWU_ERR_INVALID_ARG;    // (an empty tensor has no address)
    if (out_dtype != 0 && out_dtype != 1) return MWU_ERR_INVALID_ARG;
    if (groups <= 0 || groups > MWU_MAX_GROUPS || rows <= 0 || cols <= 0 || ldw < cols || ldi < red || ldo < features) return MWU_ERR_SHAPE;
    if (rows > MWU_MAX_GROUPED_SIDE || cols > MWU_MAX_GROUPED_SIDE || M >= (int64_t(1) << 31) - 256) return MWU_ERR_SHAPE;
    if (ldw >= (int64_t(1) << 31) || ldi >= (int64_t(1) << 31) || ldo >= (int64_t(1) << 31)) return MWU_ERR_SHAPE;
    if (w_stride < rows * ldw || w_stride >= (int64_t(1) << 38)) return MWU_ERR_SHAPE;
    if (!aligned_to(Wd, 16) || !aligned_to(in, 16) || !aligned_to(out, 16) || !aligned_to(offsets, 4) || !aligned_to(dev_status, 4) ||
        ldw % 8 != 0 || w_stride % 8 != 0 || ldi % 8 != 0 || ldo % (out_dtype ? 4 : 8) != 0)
        return MWU_ERR_ALIGNMENT;
    GroupedParams p = {};
    p.offsets = offsets;
    p.out = out; p.ldo = ldo; p.out_fp32 = out_dtype;
    p.groups = (int)groups; p.M = (int)M; p.features = (int)features; p.reduction = (int)red;
    p.feature_box = features <= 32 ? 32 : features <= 64 ? 64 : 128;
    p.dev_status = dev_status;
    p.wait = wait_limits();
    const int64_t f_tiles = (features + 255) / 256;
    if ((M / 32 + (M < groups ? M : groups)) * f_tiles >= (int64_t(1) << 30)) return MWU_ERR_SHAPE;
    int sm_count = 0;
    const int rc = check_device(&sm_count);
    if (rc != MWU_OK) return rc;
    if (M == 0) return MWU_OK;
    const int64_t runs = M < groups ? M : groups;
    p.line_tile = choose_line_tile((double)M, (double)runs, 1.0, features, (double)((red + 63) / 64), out_dtype ? 1.6 : 1.2, sm_count / 2);
    const int64_t most = (M / p.line_tile + runs) * f_tiles;
    lay_out_ring(p, features <= 32 && OP == G_FORWARD ? 4096 : features <= 64 ? G_SUB : G_SIDE, boxed_lines(p.line_tile / 2) * 128, true);
    EncodeTiledFn encode = get_encode_fn();
    if (!encode) return MWU_ERR_CUDA;
    CUtensorMap tmap_f;
    LineMaps maps_l;
    if (!encode_bf16(encode, &tmap_f, Wd, cols, rows, ldw, OP == G_FORWARD ? p.feature_box : 64, groups, w_stride)) return MWU_ERR_CUDA;
    for (int b = 2; b >= 0; --b) {
        maps_l.m[b] = maps_l.m[2];                          // (a larger box than any tile takes: never used)
        if (b < 2 && p.line_tile <= (b ? 64 : 192)) continue;
        if (!encode_bf16(encode, &maps_l.m[b], in, red, M, ldi, 128 >> b, 0, 0)) return MWU_ERR_CUDA;
    }
    CUtensorMap tmap_out;
    if (!encode_out(encode, &tmap_out, out, out_dtype != 0, features, M, ldo, 0, 0)) return MWU_ERR_CUDA;
    return launch_grouped<OP>(tmap_f, maps_l, tmap_out, p, most, sm_count, (cudaStream_t)cuda_stream) == cudaSuccess ? MWU_OK : MWU_ERR_CUDA;
}

}  // namespace gemm
}  // namespace mwu

extern "C" void mwu_debug_rows_wait(int64_t limit_cycles, int64_t slot) { mwu::gemm::set_wait_limits(limit_cycles, slot); }

extern "C" int mwu_gemm_grouped(int64_t groups, int64_t rows, int64_t cols, const void *Wd, int64_t ldw, int64_t w_stride,
                                const int32_t *offsets, const void *X, int64_t M, int64_t ldx, void *Y, int64_t ldy, int32_t y_dtype,
                                uint32_t *dev_status, void *cuda_stream) {
    using namespace mwu::gemm;
    return run_lines<G_FORWARD>(groups, rows, cols, Wd, ldw, w_stride, offsets, X, M, ldx, Y, ldy, y_dtype, dev_status, cuda_stream);
}

extern "C" int mwu_gemm_grouped_dx(int64_t groups, int64_t rows, int64_t cols, const void *Wd, int64_t ldw, int64_t w_stride,
                                   const int32_t *offsets, const void *dY, int64_t M, int64_t lddy, void *dX, int64_t lddx,
                                   int32_t dx_dtype, uint32_t *dev_status, void *cuda_stream) {
    using namespace mwu::gemm;
    return run_lines<G_DX>(groups, rows, cols, Wd, ldw, w_stride, offsets, dY, M, lddy, dX, lddx, dx_dtype, dev_status, cuda_stream);
}

extern "C" int mwu_gemm_grouped_dw(int64_t groups, int64_t rows, int64_t cols, const int32_t *offsets, const void *dY, int64_t M,
                                   int64_t lddy, const void *X, int64_t ldx, void *dW, int64_t lddw, int64_t dw_stride,
                                   int32_t dw_dtype, int32_t accumulate, uint32_t *dev_status, void *cuda_stream) {
    using namespace mwu;
    using namespace mwu::gemm;
    if (!offsets || !dW || !dev_status || M < 0 || (M > 0 && (!dY || !X))) return MWU_ERR_INVALID_ARG;      // (an empty tensor has no address)
    if ((dw_dtype != 0 && dw_dtype != 1) || (accumulate != 0 && accumulate != 1) || (accumulate && !dw_dtype)) return MWU_ERR_INVALID_ARG;
    if (groups <= 0 || groups > MWU_MAX_GROUPS || rows <= 0 || cols <= 0 || lddy < rows || ldx < cols || lddw < cols) return MWU_ERR_SHAPE;
    if (rows > MWU_MAX_GROUPED_SIDE || cols > MWU_MAX_GROUPED_SIDE || M >= (int64_t(1) << 31) - 256) return MWU_ERR_SHAPE;
    if (lddy >= (int64_t(1) << 31) || ldx >= (int64_t(1) << 31) || lddw >= (int64_t(1) << 31)) return MWU_ERR_SHAPE;
    if (dw_stride < rows * lddw || dw_stride >= (int64_t(1) << 38)) return MWU_ERR_SHAPE;
    if (!aligned_to(dY, 16) || !aligned_to(X, 16) || !aligned_to(dW, 16) || !aligned_to(offsets, 4) || !aligned_to(dev_status, 4) ||
        lddy % 8 != 0 || ldx % 8 != 0 || lddw % (dw_dtype ? 4 : 8) != 0 || dw_stride % (dw_dtype ? 4 : 8) != 0)
        return MWU_ERR_ALIGNMENT;
    GroupedParams p = {};
    p.offsets = offsets;
    p.out = dW; p.ldo = lddw; p.out_stride = dw_stride; p.out_fp32 = dw_dtype; p.accumulate = accumulate;
    p.groups = (int)groups; p.M = (int)M; p.features = (int)cols; p.lines = (int)rows;
    p.dev_status = dev_status;
    p.wait = wait_limits();
    if (groups * ((rows + 63) / 64) * ((cols + 255) / 256) >= (int64_t(1) << 30)) return MWU_ERR_SHAPE;
    int sm_count = 0;
    const int rc = check_device(&sm_count);
    if (rc != MWU_OK) return rc;
    p.line_tile = choose_line_tile((double)rows, 1.0, (double)groups, cols, (double)M / (64.0 * groups), dw_dtype ? 3.2 : 1.6, sm_count / 2);
    const int64_t tiles = groups * ((rows + p.line_tile - 1) / p.line_tile) * ((cols + 255) / 256);
    lay_out_ring(p, cols <= 64 ? G_SUB : G_SIDE, (p.line_tile / 2 + 63) / 64 * G_SUB, false);
    EncodeTiledFn encode = get_encode_fn();
    if (!encode) return MWU_ERR_CUDA;
    CUtensorMap tmap_f;
    LineMaps maps_l;
    const int64_t m_rows = M > 0 ? M : 1;               // no rows: the maps are never used, the gradients are zeros
    if (M == 0) X = dY = dW;                            // (a map has to name some address)
    if (!encode_bf16(encode, &tmap_f, X, cols, m_rows, ldx, 64, 0, 0) || !encode_bf16(encode, &maps_l.m[0], dY, rows, m_rows, lddy, 64, 0, 0))
        return MWU_ERR_CUDA;
    maps_l.m[1] = maps_l.m[2] = maps_l.m[0];
    CUtensorMap tmap_out;
    if (!encode_out(encode, &tmap_out, dW, dw_dtype != 0, cols, rows, lddw, groups, dw_stride)) return MWU_ERR_CUDA;
    return launch_grouped<G_DW>(tmap_f, maps_l, tmap_out, p, tiles, sm_count, (cudaStream_t)cuda_stream) == cudaSuccess ? MWU_OK : MWU_ERR_CUDA;
}
