// mwu_adapters_add: low-rank adapters of many requests beside a shared projection,
//
//   Y[m] = Y0[m] + s_a (X[m] . A_a^T) . B_a^T        a = the adapter of the segment that row m lies in
//
// with A_a [rank][cols], B_a [rows][rank], segments (requests) of any length.  Everything about it is bytes: the adapters in
// use, X and Y0 in, Y out, 2 * rank products to a byte or less.  Both products run in one kernel, so T = X . A^T never
// goes to memory.  CTAs of a cluster share the reduction of the first product (a slice of cols each), add up T through
// distributed shared memory, and share the columns of the second (a slice of rows of B each); T is held in fp32 and enters the
// second product as two bf16 terms, three where Y is fp32 (which leave out 2^-17, 2^-25 of it), so that only Y's own rounding shows.
//
// Segments of up to FEW_ROWS rows (generation) and longer ones (prompts) take different kernels (up to FEW_IN_ALL rows in all, the first), both decide on the
// device which segments are theirs, and where both are launched they run at the same time:
//   mwu_adapters_few_kernel   16 rows of an adapter (of a segment, in batches that are not sorted: an adapter is then read once a
//                             segment) to a cluster of 2 to 8 CTAs, mma.sync straight from global memory (an item reads its operands
//                             once and the tensor work is nothing; a lane's eight consecutive elements stand for a permuted reduction order)
//   mwu_adapters_tile_kernel  128 rows to a cluster of 1 to 8 CTAs, TMA and tcgen05.mma, Y0 and Y through shared memory
//
// What bounds them (us a call among others).  Few rows: latency.  One row, rank 16, 4096 -> 4096: 5 on the device (list 1.1, first product 0.7, adding
// it up 1.7, second 0.8), 9.5 with the host.  64 rows of 32 adapters, rank 32, 4096 -> 16384: 17.4 (3 to sort, 2.5, 3, 5); 73 before loads stood ahead of
// tests of their values, 35 before rows were sorted by adapter, 19 with one run of columns at a time; B and Y0 brought to L2 ahead: no
// faster, and 1 us to ask for.  Many rows: three phases one after another.  8192 rows, rank 64, 4096 -> 4096: 46.0 (X in at 4.1 TB/s, 5 us to add
// up T, Y0 in and Y out at 5.4; the tiles that end inside 32 rows, whose boxes leave by plain stores, end last: 49.9 with one store to a lane at a time).
// Rows without an adapter are copied with eight loads in flight (one: 72 instead of 45 us for that tile).
//
// Every wait on an mbarrier is bounded; when one runs out the kernel raises MWU_DEV_TIMEOUT, waits for its copies in
// flight, frees tensor memory and returns.
#include "mwu_rows.cuh"

namespace mwu {
namespace gemm {
EncodeTiledFn get_encode_fn();          // mwu_gemm.cu
}  // namespace gemm

namespace adapters {
using namespace gemm;

constexpr int FEW_ROWS = 32;            // rows of a segment that the first kernel takes,
constexpr int FEW_IN_ALL = 256;         // rows of a call that it takes whatever its segments,
constexpr int SORTED_ROWS = 512;        // and rows of a call that it sorts by adapter: as many as sort_rows has place for
constexpr int FEW_THREADS = 256;
constexpr int TILE_THREADS = 320;
constexpr int TILE_ROWS = 128;          // rows of an item of the tile kernel

struct Params {
    const __nv_bfloat16 *A, *B, *X;
    long long lda, a_stride, ldb, b_stride, ldx, ldy;
    const float *scale;
    const int *offsets, *which;
    const void *Y0;
    void *Y;
    int adapters, rank, rows, cols, segments, M;
    int few_rows;                       // FEW_ROWS, or as many as may be
    int sorted;                         // the few-rows kernel's rows are sorted by adapter
    int beside;                         // the few-rows kernel runs beside the tile kernel launched before it
    WaitLimits wait;                    // of the tile kernel
    unsigned *dev_status;
};

// ------------------------------------------------------------------------------------------
// which rows a cluster works on
// ------------------------------------------------------------------------------------------
struct Finder {
    int warp_sum[32];
    int item, row0, count, adapter;
};

// rows of a segment that lie in one work item, or 0 where the segment is the other kernel's
template <bool FEW>
__device__ __forceinline__ int item_rows(const Params &p, int len) { return (len <= p.few_rows) == FEW ? (FEW ? 16 : TILE_ROWS) : 0; }

// Thread i looks after segments i * per .. of the list; its items are number `first` and on.  Returns how many there are in all,
// -1 where the list makes no sense.  All threads of the CTA.
template <bool FEW, int THREADS>
__device__ __forceinline__ int count_items(const Params &p, Finder *f, int per, int &first) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, s0 = threadIdx.x * per;
    int bad = 0, mine = 0;
    for (int s = s0; s < s0 + per && s < p.segments; ++s) {
        const int a = __ldg(p.offsets + s), b = __ldg(p.offsets + s + 1), w = __ldg(p.which + s);
        const bool wrong = a < 0 || b < a || b > p.M || w < -1 || w >= p.adapters;
        bad |= wrong;
        const int unit = wrong ? 0 : item_rows<FEW>(p, b - a);
        if (unit) mine += (b - a + unit - 1) / unit;
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) f->warp_sum[warp] = upto;
    bad = __syncthreads_or(bad);
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const int v = f->warp_sum[w];
        if (w < warp) before += v;
        total += v;
    }
    first = before + upto - mine;
    return bad ? -1 : total;
}

// the thread that looks after item `item` says where it is; the others read it behind the barrier that follows
template <bool FEW>
__device__ __forceinline__ void find_item(const Params &p, Finder *f, int per, int first, int item) {
    if (item < first) return;
    int at = first;
    for (int s = threadIdx.x * per; s < (int)(threadIdx.x + 1) * per && s < p.segments; ++s) {
        const int a = __ldg(p.offsets + s), len = __ldg(p.offsets + s + 1) - a, unit = item_rows<FEW>(p, len);
        const int n = unit ? (len + unit - 1) / unit : 0;
        if (item < at + n) {
            const int r = (item - at) * unit;
            f->row0 = a + r;
            f->count = min(unit, len - r);
            f->adapter = __ldg(p.which + s);
            return;
        }
        at += n;
    }
}

// Up to SORTED_ROWS rows of a call are worked on adapter by adapter, 16 rows at a time, wherever in the batch they are: 64 tokens of 32
// adapters read every adapter once, not twice (4096 -> 16384: 17 us instead of 35), and 512 tokens of 4 adapters once for 16 rows.
struct Sorter {
    alignas(16) int key[SORTED_ROWS];   // adapter of a row; NOBODY: not this kernel's (read 16 bytes at a time)
    int row[SORTED_ROWS];               // rows in the order of their adapters
    int start[SORTED_ROWS + 1];         // where an item's rows start in `row`
    unsigned starts[SORTED_ROWS / 32];
    int counted;
};
static_assert(alignof(Sorter) == 16 && SORTED_ROWS % 4 == 0, "adapters: keys are read in fours");
constexpr int NOBODY = 0x7fffffff;

// Returns the number of items, -1 where the list makes no sense.  All threads of the CTA, each placing two rows by counting those that
// come before them, which takes the square of the rows: up to all that the arrays hold, sorted is the faster.  (A bitonic sort is a
// barrier a step: 3.4 us more for 64 rows.  Single tokens, 4 adapters, rank 32, 4096 -> 16384, sorted / segment by segment: 257 rows
// 25 us / 64, 384 34 / 94, 512 52 / 114.)
__device__ __forceinline__ int sort_rows(const Params &p, Sorter *o, int per) {
    constexpr int MINE = SORTED_ROWS / FEW_THREADS;
    const int tid = threadIdx.x;
#pragma unroll
    for (int q = 0; q < MINE; ++q) o->key[tid + q * FEW_THREADS] = NOBODY;
    if (tid < SORTED_ROWS / 32) o->starts[tid] = 0u;
    if (tid == 0) o->counted = 0;
    __syncthreads();
    int bad = 0, rows = 0;
    for (int s = tid * per; s < (tid + 1) * per && s < p.segments; ++s) {
        const int a = __ldg(p.offsets + s), b = __ldg(p.offsets + s + 1), w = __ldg(p.which + s);
        const bool wrong = a < 0 || b < a || b > p.M || w < -1 || w >= p.adapters;
        bad |= wrong;
        if (!wrong && b - a <= p.few_rows) {
            rows += b - a;
            for (int r = a; r < b; ++r) o->key[r] = w;
        }
    }
    if (rows) atomicAdd(&o->counted, rows);
    if (__syncthreads_or(bad)) return -1;
    if (o->counted == 0) return 0;                          // all of them the other kernel's
    int at[MINE];
    bool first[MINE];
#pragma unroll
    for (int q = 0; q < MINE; ++q) {
        const int r = tid + q * FEW_THREADS, mine = o->key[r];
        int less = 0, same = 0;                             // rows of smaller adapters; of mine, before this one
        if (mine != NOBODY)
            for (int j = 0; j < p.M; j += 4) {
                const int4 k = *reinterpret_cast<const int4 *>(&o->key[j]);
                less += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
                same += (k.x == mine && j < r) + (k.y == mine && j + 1 < r) + (k.z == mine && j + 2 < r) + (k.w == mine && j + 3 < r);
            }
        at[q] = less + same;
        first[q] = mine != NOBODY && same % 16 == 0;
        if (mine != NOBODY) o->row[at[q]] = r;
        if (first[q]) atomicOr(&o->starts[at[q] / 32], 1u << (at[q] % 32));
    }
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < SORTED_ROWS / 32; ++w) total += __popc(o->starts[w]);
#pragma unroll
    for (int q = 0; q < MINE; ++q)
        if (first[q]) {
            int before = __popc(o->starts[at[q] / 32] & ((1u << (at[q] % 32)) - 1u));
            for (int w = 0; w < at[q] / 32; ++w) before += __popc(o->starts[w]);
            o->start[before] = at[q];
        }
    if (tid == 0) o->start[total] = o->counted;
    __syncthreads();
    return total;
}

// Y = Y0 (or zeros) for rows without an adapter, columns n0 .. n1 (n0 a multiple of 32): a row to a warp, 16 bytes to a lane, AT_ONCE of
// them in flight
template <bool F32, int AT_ONCE, typename RowOf>
__device__ __forceinline__ void copy_rows(const Params &p, RowOf row_of, int count, int n0, int n1, int warp, int warps) {
    if (p.Y0 == p.Y || n1 <= n0) return;
    constexpr int SIZE = F32 ? 4 : 2, UNIT = 16 / SIZE;
    const int lane = threadIdx.x & 31, whole = (n1 - n0) / UNIT;
#pragma unroll 1
    for (int r = warp; r < count; r += warps) {
        const long long at = ((long long)row_of(r) * p.ldy + n0) * SIZE;
        const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned char *>(p.Y0) + at);
        uint4 *to = reinterpret_cast<uint4 *>(reinterpret_cast<unsigned char *>(p.Y) + at);
#pragma unroll 1
        for (int u = lane; u < whole; u += 32 * AT_ONCE) {
            uint4 v[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                v[j] = make_uint4(0, 0, 0, 0);
                if (p.Y0 && u + 32 * j < whole) v[j] = from[u + 32 * j];
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (u + 32 * j < whole) to[u + 32 * j] = v[j];
        }
        const int e = whole * UNIT + lane;                  // the last few elements
        if (e < n1 - n0) {
            if (F32) reinterpret_cast<unsigned *>(to)[e] = p.Y0 ? reinterpret_cast<const unsigned *>(from)[e] : 0u;
            else reinterpret_cast<unsigned short *>(to)[e] = p.Y0 ? reinterpret_cast<const unsigned short *>(from)[e] : (unsigned short)0;
        }
    }
}

// ------------------------------------------------------------------------------------------
// few rows
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_16816(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Loads come first and what lies past the end of a row is cleared afterwards, and only where a row ends: a test that
// needs the value of one load would hold up the next.
__device__ __forceinline__ uint4 load8_if(const __nv_bfloat16 *at, bool take) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (take) v = __ldg(reinterpret_cast<const uint4 *>(at));
    return v;
}
__device__ __forceinline__ uint2 load4_if(const __nv_bfloat16 *at, bool take) {
    uint2 v = make_uint2(0, 0);
    if (take) v = __ldg(reinterpret_cast<const uint2 *>(at));
    return v;
}
// the first `valid` of a word's two halves of elements e, e + 1
__device__ __forceinline__ unsigned keep_valid(unsigned w, int e, int valid) {
    return e + 1 < valid ? w : (e < valid ? w & 0xffffu : 0u);
}
__device__ __forceinline__ void keep8(uint4 &v, int valid) {
    v.x = keep_valid(v.x, 0, valid);
    v.y = keep_valid(v.y, 2, valid);
    v.z = keep_valid(v.z, 4, valid);
    v.w = keep_valid(v.w, 6, valid);
}
// The next bf16 terms of two numbers, and the numbers without them.  All terms but the last stop at the largest bf16: a number that would
// round to an infinity keeps a finite remainder, and an infinity goes whole into the last term (inf - inf would make NaN of it).
template <bool LAST>
__device__ __forceinline__ unsigned next_terms(float &lo, float &hi) {
    unsigned w;
    if (LAST) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    lo -= __uint_as_float(w << 16);
    hi -= __uint_as_float(w & 0xffff0000u);
    return w;
}
__device__ __forceinline__ float remote_f32(unsigned local, unsigned cta) {
    unsigned at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(local), "r"(cta));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ unsigned cluster_size() {
    unsigned n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}


template <int R, bool F32>
struct Few {
    static constexpr int TERMS = F32 ? 3 : 2;
    static constexpr int T_LD = R + 8;                      // elements of a row of T: the eight rows of a load fall into different banks
    float red[FEW_THREADS / 64][16][R];
    float part[16][R];
    __nv_bfloat16 T[TERMS][16][T_LD];
};

// 16 rows of one adapter or segment to a cluster.  First product: CTA c of the cluster takes its share of cols in chunks of 32, a warp a
// chunk at a time: lane (g, t) = (lane / 4, lane % 4) loads elements 8t .. 8t + 7 of the chunk of rows g and g + 8 of X and of rows
// 8i + g of A, 16 bytes each, and the two MMAs of a chunk take words 0, 1 and 2, 3 of both: the order of the reduction is
// permuted alike in both operands.  Second product: 32 columns of Y at a time, MMA i multiplying with rows
// 8(g / 2) + 2i + g % 2 of B, which leaves lane (g, t) with eight consecutive columns of rows g and g + 8.
template <int R, bool F32>
__global__ void __launch_bounds__(FEW_THREADS, R <= 64 ? 2 : 1)
mwu_adapters_few_kernel(const Params p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ union { Finder f; Sorter o; } find;
    Finder &f = find.f;
    Few<R, F32> *sm = reinterpret_cast<Few<R, F32> *>(smem_raw);
    constexpr int TERMS = Few<R, F32>::TERMS;
    // Beside the tile kernel: that one has waited for what came before it, so the inputs are there; its own rows are others than these.
    if (!p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int c = (int)cluster_rank(), ctas = (int)cluster_size(), clusters = (int)gridDim.x / ctas;
    const int per = (p.segments + FEW_THREADS - 1) / FEW_THREADS;
    int first = 0;
    const int total = p.sorted ? sort_rows(p, &find.o, per) : count_items<true, FEW_THREADS>(p, &f, per, first);
    if (total < 0 && blockIdx.x == 0 && tid == 0) atomicOr(p.dev_status, (unsigned)MWU_DEV_BOUNDS);
    const int k_chunks = (p.cols + 31) / 32, n_groups = (p.rows + 31) / 32;
    const int kc0 = (int)((long long)k_chunks * c / ctas), kc1 = (int)((long long)k_chunks * (c + 1) / ctas);
    const int ng0 = (int)((long long)n_groups * c / ctas), ng1 = (int)((long long)n_groups * (c + 1) / ctas);

    for (int item = (int)blockIdx.x / ctas; item < total; item += clusters) {
        int row0 = 0, count, a;
        const int *rows = nullptr;
        if (p.sorted) {
            const int at = find.o.start[item];
            count = find.o.start[item + 1] - at;
            rows = &find.o.row[at];
            a = find.o.key[rows[0]];
        } else {
            __syncthreads();
            find_item<true>(p, &f, per, first, item);
            __syncthreads();
            row0 = f.row0;
            count = f.count;
            a = f.adapter;
        }
        auto row_of = [&](int r) { return rows ? rows[r] : row0 + r; };
        if (a < 0) {
            copy_rows<F32, 2>(p, row_of, count, ng0 * 32, min(p.rows, ng1 * 32), warp, FEW_THREADS / 32);
            continue;
        }
        // this lane's two rows (the first one again where there are fewer: read, never written)
        const long long r0 = row_of(g < count ? g : 0), r1 = row_of(g + 8 < count ? g + 8 : 0);
        // ---- T = X . A^T over this CTA's slice of cols ----
        // Sums leave the tensor core every 512 products of a warp, as in the kernel for many rows: it drops what lies below an
        // accumulator's last place, always towards zero (6e-5 of a sum of 65536 products in one piece).
        constexpr int PIECE = 512 / 32 * (FEW_THREADS / 32);    // chunks of the CTA: up to 8192 columns of two CTAs, one piece
        const __nv_bfloat16 *x0 = p.X + r0 * p.ldx + 8 * t, *x1 = p.X + r1 * p.ldx + 8 * t;
        const __nv_bfloat16 *a0 = p.A + (long long)a * p.a_stride + (long long)g * p.lda + 8 * t;
        constexpr int BATCH = R / 8 < 8 ? R / 8 : 8;        // loads of A in flight, of each of
        constexpr int AHEAD = R <= 32 ? 2 : 1;              // so many chunks
        int piece = kc0;
        do {
            float acc[R / 8][4];
#pragma unroll
            for (int i = 0; i < R / 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
            const int end = min(kc1, piece + PIECE);
            for (int ch = piece + warp; ch < end; ch += AHEAD * (FEW_THREADS / 32)) {
                uint4 u[AHEAD], v[AHEAD], w[AHEAD][BATCH];
#pragma unroll
                for (int i0 = 0; i0 < R / 8; i0 += BATCH) {
#pragma unroll
                    for (int h = 0; h < AHEAD; ++h) {
                        const int cc = ch + h * (FEW_THREADS / 32), k = cc * 32, valid = cc < end ? p.cols - k - 8 * t : 0;
                        if (i0 == 0) {
                            u[h] = load8_if(x0 + k, g < count && valid > 0);
                            v[h] = load8_if(x1 + k, g + 8 < count && valid > 0);
                        }
#pragma unroll
                        for (int i = 0; i < BATCH; ++i)
                            w[h][i] = load8_if(a0 + (long long)(8 * (i0 + i)) * p.lda + k, 8 * (i0 + i) + g < p.rank && valid > 0);
                    }
#pragma unroll
                    for (int h = 0; h < AHEAD; ++h) {
                        const int k = (ch + h * (FEW_THREADS / 32)) * 32, valid = p.cols - k - 8 * t;
                        if (p.cols - k < 32) {
                            keep8(u[h], valid);
                            keep8(v[h], valid);
#pragma unroll
                            for (int i = 0; i < BATCH; ++i) keep8(w[h][i], valid);
                        }
#pragma unroll
                        for (int i = 0; i < BATCH; ++i) {
                            mma_16816(acc[i0 + i], u[h].x, v[h].x, u[h].y, v[h].y, w[h][i].x, w[h][i].y);
                            mma_16816(acc[i0 + i], u[h].z, v[h].z, u[h].w, v[h].w, w[h][i].z, w[h][i].w);
                        }
                    }
                }
            }
            // the warps' sums, the upper four onto the lower four first: half the memory; onto those of the pieces before
            float2 *mine = reinterpret_cast<float2 *>(&sm->red[warp % (FEW_THREADS / 64)][g][2 * t]);
#pragma unroll
            for (int up = 1; up >= 0; --up) {
                if (warp / (FEW_THREADS / 64) == up) {
#pragma unroll
                    for (int i = 0; i < R / 8; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float2 *at = mine + h * 4 * R + 4 * i;          // eight rows on, eight ranks on
                            float2 v = make_float2(acc[i][2 * h], acc[i][2 * h + 1]);
                            if (up == 0 || piece > kc0) {
                                const float2 o = *at;
                                v.x += o.x;
                                v.y += o.y;
                            }
                            *at = v;
                        }
                }
                __syncthreads();
            }
            piece += PIECE;
        } while (piece < kc1);
        for (int e = tid; e < 16 * R; e += FEW_THREADS) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < FEW_THREADS / 64; ++w) s += (&sm->red[w][0][0])[e];
            (&sm->part[0][0])[e] = s;
        }
        cluster_arrive();
        // the operands of this warp's first columns travel meanwhile
        const __nv_bfloat16 *b0 = p.B + (long long)a * p.b_stride + (R >= 32 ? 8 : 4) * t;
        constexpr int WIDE = R >= 32 ? 32 : 16;             // ranks of a load of the warp: 16 or 8 bytes a lane
        constexpr int AT_ONCE = R <= 32 ? 2 : 1;            // runs of 32 columns a warp has under way
        constexpr int STEP = AT_ONCE * (FEW_THREADS / 32);
        uint4 w[AT_ONCE][4][R / WIDE];
        uint4 y0[AT_ONCE][2][F32 ? 2 : 1];
        auto load_groups = [&](int grp0) {
#pragma unroll
            for (int z = 0; z < AT_ONCE; ++z) {
                const int grp = grp0 + z * (FEW_THREADS / 32);
                const bool here = grp < ng1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = grp * 32 + 8 * (g >> 1) + 2 * i + (g & 1);
#pragma unroll
                    for (int s = 0; s < R / WIDE; ++s) {
                        const __nv_bfloat16 *at = b0 + (long long)n * p.ldb + WIDE * s;
                        if constexpr (R >= 32) {
                            w[z][i][s] = load8_if(at, here && n < p.rows && 32 * s + 8 * t < p.rank);
                        } else {
                            const uint2 v = load4_if(at, here && n < p.rows && 4 * t < p.rank);
                            w[z][i][s] = make_uint4(v.x, v.y, 0, 0);
                        }
                    }
                }
                const int n = grp * 32 + 8 * t;
                const unsigned char *from = reinterpret_cast<const unsigned char *>(p.Y0);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < (F32 ? 2 : 1); ++e) {
                        y0[z][h][e] = make_uint4(0, 0, 0, 0);
                        if (p.Y0 && here && g + 8 * h < count && n + 8 <= p.rows)
                            y0[z][h][e] = *reinterpret_cast<const uint4 *>(from + ((h ? r1 : r0) * p.ldy + n) * (F32 ? 4 : 2) + 16 * e);
                    }
            }
        };
        load_groups(ng0 + warp);
        cluster_wait();
        // ---- the cluster's sum, scaled, as bf16 terms ----
        const float scale = p.scale ? __ldg(p.scale + a) : 1.f;
        for (int e = tid; e < 16 * R; e += FEW_THREADS) {
            float s = 0.f, none = 0.f;
#pragma unroll 4
            for (int o = 0; o < ctas; ++o) s += remote_f32(smem_u32(&(&sm->part[0][0])[e]), (unsigned)o);
            s *= scale;
            if (e % R >= p.rank) s = 0.f;                   // (an infinity of X times the zeros that stand for A there is NaN)
#pragma unroll
            for (int q = 0; q < TERMS; ++q)
                reinterpret_cast<unsigned short &>(sm->T[q][e / R][e % R]) = (unsigned short)(q + 1 < TERMS ? next_terms<false>(s, none) : next_terms<true>(s, none));
        }
        cluster_arrive();                                   // the others' sums have been read; waited for below
        __syncthreads();
        // ---- Y = Y0 + T . B^T over this CTA's slice of rows ----
        for (int grp0 = ng0 + warp; grp0 < ng1; grp0 += STEP) {
          float d[AT_ONCE][4][4];
#pragma unroll
          for (int z = 0; z < AT_ONCE; ++z) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) d[z][i][j] = 0.f;
            if (p.rank & (R >= 32 ? 7 : 3)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int s = 0; s < R / WIDE; ++s) keep8(w[z][i][s], p.rank - WIDE * s - (R >= 32 ? 8 : 4) * t);
            }
          }
#pragma unroll
          for (int s = 0; s < R / WIDE; ++s)
#pragma unroll
            for (int q = TERMS - 1; q >= 0; --q) {
                if constexpr (R >= 32) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(&sm->T[q][g][32 * s + 8 * t]);
                    const uint4 v = *reinterpret_cast<const uint4 *>(&sm->T[q][g + 8][32 * s + 8 * t]);
#pragma unroll
                    for (int z = 0; z < AT_ONCE; ++z)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            mma_16816(d[z][i], u.x, v.x, u.y, v.y, w[z][i][s].x, w[z][i][s].y);
                            mma_16816(d[z][i], u.z, v.z, u.w, v.w, w[z][i][s].z, w[z][i][s].w);
                        }
                } else {
                    const uint2 u = *reinterpret_cast<const uint2 *>(&sm->T[q][g][4 * t]);
                    const uint2 v = *reinterpret_cast<const uint2 *>(&sm->T[q][g + 8][4 * t]);
#pragma unroll
                    for (int z = 0; z < AT_ONCE; ++z)
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma_16816(d[z][i], u.x, v.x, u.y, v.y, w[z][i][s].x, w[z][i][s].y);
                }
            }
#pragma unroll
          for (int z = 0; z < AT_ONCE; ++z) {
            const int grp = grp0 + z * (FEW_THREADS / 32);
            if (grp >= ng1) break;
            const int n = grp * 32 + 8 * t, left = p.rows - n;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (g + 8 * h >= count || left <= 0) continue;
                const long long at = (h ? r1 : r0) * p.ldy + n;
                const unsigned in[8] = {y0[z][h][0].x, y0[z][h][0].y, y0[z][h][0].z, y0[z][h][0].w, y0[z][h][F32].x, y0[z][h][F32].y, y0[z][h][F32].z, y0[z][h][F32].w};
                if (F32) {
                    float *y = reinterpret_cast<float *>(p.Y) + at;
                    if (left >= 8) {
                        float o[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = __uint_as_float(in[j]) + d[z][j / 2][2 * h + j % 2];
                        *reinterpret_cast<float4 *>(y) = make_float4(o[0], o[1], o[2], o[3]);
                        *reinterpret_cast<float4 *>(y + 4) = make_float4(o[4], o[5], o[6], o[7]);
                    } else {
                        const float *b = reinterpret_cast<const float *>(p.Y0) + at;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (j < left) y[j] = (p.Y0 ? b[j] : 0.f) + d[z][j / 2][2 * h + j % 2];
                    }
                } else {
                    __nv_bfloat16 *y = reinterpret_cast<__nv_bfloat16 *>(p.Y) + at;
                    if (left >= 8) {
                        unsigned out[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 o = __floats2bfloat162_rn(__uint_as_float(in[i] << 16) + d[z][i][2 * h],
                                                                           __uint_as_float(in[i] & 0xffff0000u) + d[z][i][2 * h + 1]);
                            out[i] = *reinterpret_cast<const unsigned *>(&o);
                        }
                        *reinterpret_cast<uint4 *>(y) = make_uint4(out[0], out[1], out[2], out[3]);
                    } else {
                        const __nv_bfloat16 *b = reinterpret_cast<const __nv_bfloat16 *>(p.Y0) + at;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (j < left) y[j] = __float2bfloat16_rn((p.Y0 ? __bfloat162float(b[j]) : 0.f) + d[z][j / 2][2 * h + j % 2]);
                    }
                }
            }
          }
          load_groups(grp0 + STEP);
        }
        cluster_wait();
    }
    if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");      // what comes behind this kernel comes behind both
}

// ------------------------------------------------------------------------------------------
// many rows
// ------------------------------------------------------------------------------------------
// A stage of the first product: 128 rows x 64 columns of X and R x 64 of A.  A chunk of the second: 128 rows x 128 bytes of Y0
// (64 columns of bf16, 32 of fp32) and as many rows of B.  Both go through the same ring of slots, so the first chunks of Y0 and B come
// in while T is still being added up, and the next item's first stages while this one's last chunks leave.
// (Items of 64 rows, a CTA to each and nothing to add up between CTAs: 76 us instead of 54 for 8192 rows, 4096 -> 4096, rank 64; a
// step of either product takes 0.3 to 0.5 us however few rows it has.)
// This kernel's clusters hold tensor memory while their CTAs wait for one another.  Were a CTA of another such kernel (on another
// stream) on the same SM, each could hold what the other waits for; with this much shared memory none fits beside it (the least
// that such a kernel takes is 36 KB).
constexpr int TILE_SMEM = 196 * 1024;
constexpr int TILE_SLOTS = 8;           // most slots of a ring
constexpr int TILE_ITEMS = 64;          // most items of a cluster

template <int R, bool F32>
struct TileCfg {
    static constexpr int TERMS = F32 ? 3 : 2;
    static constexpr int CW = F32 ? 32 : 64;                // columns of Y in a chunk
    static constexpr int BLOCKS = R > 64 ? 2 : 1;           // 64 ranks to a 128-byte row
    static constexpr int ROWS_BYTES = TILE_ROWS * 128;
    static constexpr int OPERAND = 8192 * BLOCKS;           // of A or B in a slot
    static constexpr int T_BYTES = TERMS * BLOCKS * ROWS_BYTES;
    static constexpr bool POW2 = R > 64 && F32;             // only clusters of 1, 2, 4 or 8 fit
    static constexpr int SUM_BYTES = (POW2 ? 128 : 133) * R * 4;    // of at most 8 CTAs' shares of 128 rows, each rounded up
    static constexpr int EXTRA = 1024 + 2048;               // alignment, and what TileSmem takes
    static constexpr int SMEM = R > 64 ? 227 * 1024 : TILE_SMEM;
    static constexpr int SLOT = ROWS_BYTES + OPERAND;
    static constexpr int ALONE = (SMEM - EXTRA - T_BYTES) / SLOT, TOGETHER = (SMEM - EXTRA - T_BYTES - SUM_BYTES) / SLOT;   // slots of a CTA
    static_assert(ALONE <= TILE_SLOTS && TOGETHER >= 2, "adapter tile kernel: slots");
};

struct TileSmem {
    unsigned long long full[TILE_SLOTS], empty[TILE_SLOTS], tfull1[2], tempty1[2], tfull2[2], tempty2[2], drain;
    unsigned tmem_base;
    int abort, drain_abort;
    int row0[TILE_ITEMS], count[TILE_ITEMS], adapter[TILE_ITEMS];
    Finder f;
};
static_assert(sizeof(TileSmem) <= 2048, "adapter tile kernel: shared memory");

__device__ __forceinline__ void tma_load_3d(unsigned dst, const CUtensorMap *map, unsigned bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// place in a ring of slots: the slot and how often the ring has been gone round, for its parity
struct Place {
    int slot = 0;
    unsigned round = 0;
    __device__ __forceinline__ void advance(int by, int slots) {            // by <= slots
        slot += by;
        if (slot >= slots) { slot -= slots; ++round; }
    }
    __device__ __forceinline__ void retreat(int slots) {
        if (--slot < 0) { slot += slots; --round; }
    }
};

// items cluster, cluster + clusters, ... into the list, by the threads that look after them
__device__ __forceinline__ void list_items(const Params &p, TileSmem *sm, int per, int first, int cluster, int clusters) {
    int at = first;
    for (int s = threadIdx.x * per; s < (int)(threadIdx.x + 1) * per && s < p.segments; ++s) {
        const int a = __ldg(p.offsets + s), len = __ldg(p.offsets + s + 1) - a, unit = item_rows<false>(p, len);
        const int n = unit ? (len + unit - 1) / unit : 0;
        for (int i = at <= cluster ? cluster : cluster + (at - cluster + clusters - 1) / clusters * clusters; i < at + n; i += clusters) {
            const int k = (i - cluster) / clusters, r = (i - at) * unit;
            sm->row0[k] = a + r;
            sm->count[k] = min(unit, len - r);
            sm->adapter[k] = __ldg(p.which + s);
        }
        at += n;
    }
}

template <int R, bool F32>
__global__ void __launch_bounds__(TILE_THREADS, 1)
mwu_adapters_tile_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_a,
                         const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_y0,
                         const __grid_constant__ CUtensorMap tm_y, const __grid_constant__ Params p) {
    using C = TileCfg<R, F32>;
    extern __shared__ unsigned char smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ctas = (int)cluster_size(), c = (int)cluster_rank();
    const int slots = ctas > 1 ? C::TOGETHER : C::ALONE;
    unsigned char *ring = smem_raw + smem_pad_1024(smem_raw);
    unsigned char *sT = ring + slots * C::SLOT;
    float4 *sums = reinterpret_cast<float4 *>(sT + C::T_BYTES);
    TileSmem *sm = reinterpret_cast<TileSmem *>(ring + C::SMEM - C::EXTRA);
    volatile int *abort = &sm->abort;

    if (threadIdx.x == 0) {
        for (int s = 0; s < TILE_SLOTS; ++s) {
            mbar_init(smem_u32(&sm->full[s]), 1 + (s == p.wait.dead_slot));
            mbar_init(smem_u32(&sm->empty[s]), 4);          // the four warps of a chunk; a stage's MMAs arrive for all four
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sm->tfull1[b]), 1);
            mbar_init(smem_u32(&sm->tempty1[b]), 8);
            mbar_init(smem_u32(&sm->tfull2[b]), 1);
            mbar_init(smem_u32(&sm->tempty2[b]), 4);
        }
        mbar_init(smem_u32(&sm->drain), 1);
        sm->abort = 0;
        sm->drain_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 1) {
        tmem_alloc(smem_u32(&sm->tmem_base), 512);
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the kernel for few rows works beside this one
    }
    const int per = (p.segments + TILE_THREADS - 1) / TILE_THREADS;
    int first;
    const int total = count_items<false, TILE_THREADS>(p, &sm->f, per, first);
    const int cluster = (int)blockIdx.x / ctas, clusters = (int)gridDim.x / ctas;
    if (total > 0) list_items(p, sm, per, first, cluster, clusters);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem_base = *reinterpret_cast<volatile unsigned *>(&sm->tmem_base);
    const int items = total > cluster ? (total - cluster + clusters - 1) / clusters : 0;    // the whole cluster alike
    const int k_all = (p.cols + 63) / 64, n_all = (p.rows + C::CW - 1) / C::CW;
    const int ks0 = (int)((long long)k_all * c / ctas), ks1 = (int)((long long)k_all * (c + 1) / ctas);
    const int nc0 = (int)((long long)n_all * c / ctas), nc1 = (int)((long long)n_all * (c + 1) / ctas);
    constexpr int PIECE = 8;                                // stages between two sums of T (512 products)

    // For every item all threads of the cluster meet three times: when all CTAs are done with the item before (1), when the sums
    // have been given to their owners (2), and when T is with everybody (3).  Every role passes them whether a wait of its own ran
    // out or not.
    if (warp == 0) {
        // ---------------- TMA producer ----------------
        bool ok = true;
        Place at;
#pragma unroll 1
        for (int it = 0; it < items; ++it) {
            const int row0 = sm->row0[it], a = sm->adapter[it], bands = (sm->count[it] + 31) / 32;
            if (a < 0) continue;
            cluster_arrive();
            for (int ks = ks0; ok && ks < ks1; ++ks) {
                if (at.round) ok = warp_wait_spin(smem_u32(&sm->empty[at.slot]), (at.round & 1u) ^ 1u, abort, p.wait.cycles);
                if (!ok) break;
                if (elect_one()) {
                    const unsigned bar = smem_u32(&sm->full[at.slot]), dst = smem_u32(ring + at.slot * C::SLOT);
                    mbar_expect_tx(bar, (unsigned)(bands * 4096 + R * 128));
                    for (int b = 0; b < bands; ++b) tma_load_2d(dst + b * 4096, &tm_x, bar, ks * 64, row0 + 32 * b);
                    tma_load_3d(dst + C::ROWS_BYTES, &tm_a, bar, ks * 64, 0, a);
                }
                __syncwarp();
                at.advance(1, slots);
            }
            cluster_wait();                                 // (1)
            cluster_arrive();
            bool waited = false;
            for (int i = nc0; ok && i < nc1; ++i) {
                if (i - nc0 == slots) {                     // from here on a slot comes free only once T is there
                    cluster_wait();                         // (2)
                    cluster_arrive();
                    cluster_wait();                         // (3)
                    waited = true;
                }
                if (at.round) ok = warp_wait_spin(smem_u32(&sm->empty[at.slot]), (at.round & 1u) ^ 1u, abort, p.wait.cycles);
                if (!ok) break;
                if (elect_one()) {
                    const unsigned bar = smem_u32(&sm->full[at.slot]), dst = smem_u32(ring + at.slot * C::SLOT);
                    mbar_expect_tx(bar, (unsigned)((p.Y0 ? bands * 4096 : 0) + C::CW * 128 * C::BLOCKS));
                    for (int q = 0; q < C::BLOCKS; ++q)
                        tma_load_3d(dst + C::ROWS_BYTES + q * C::CW * 128, &tm_b, bar, 64 * q, i * C::CW, a);
                    if (p.Y0)
                        for (int b = 0; b < bands; ++b) tma_load_2d(dst + b * 4096, &tm_y0, bar, i * C::CW, row0 + 32 * b);
                }
                __syncwarp();
                at.advance(1, slots);
            }
            if (!waited) {
                cluster_wait();                             // (2)
                cluster_arrive();
                cluster_wait();                             // (3)
            }
        }
        // a wait ran out: the loads in flight land before this CTA leaves
        if (__any_sync(0xffffffffu, *abort)) {
            for (int s = 0; s < slots; ++s)
                if (at.round || s < at.slot)                // this slot's latest load
                    mbar_wait(smem_u32(&sm->full[s]), (s < at.slot ? at.round : at.round - 1u) & 1u, &sm->drain_abort, p.wait.cycles);
            __syncwarp();
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        bool ok = true;
        Place at;
        unsigned use = 0, used2 = 0;                        // uses of the first product's accumulators; bit b: parity of those of the second's b
#pragma unroll 1
        for (int it = 0; it < items; ++it) {
            if (sm->adapter[it] < 0) continue;
            cluster_arrive();
            for (int k0 = ks0; ok && k0 < ks1; k0 += PIECE, ++use) {
                ok = warp_wait_spin(smem_u32(&sm->tempty1[use & 1u]), ((use >> 1) & 1u) ^ 1u, abort, p.wait.cycles);
                if (!ok) break;
                tc_fence_after();
                const int k1 = min(ks1, k0 + PIECE);
                for (int ks = k0; ks < k1; ++ks, at.advance(1, slots)) {
                    const int s = at.slot;
                    ok = warp_wait_spin(smem_u32(&sm->full[s]), at.round & 1u, abort, p.wait.cycles);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const unsigned long long xd = make_desc(smem_u32(ring + s * C::SLOT));
                        const unsigned long long ad = make_desc(smem_u32(ring + s * C::SLOT + C::ROWS_BYTES));
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4)
                            umma_bf16(tmem_base + (use & 1u) * R, xd + 2ull * k4, ad + 2ull * k4, make_idesc(R), (ks > k0 || k4) ? 1u : 0u);
                        for (int i = 0; i < 3; ++i) mbar_arrive(smem_u32(&sm->empty[s]));
                        umma_commit(smem_u32(&sm->empty[s]));
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (elect_one()) umma_commit(smem_u32(&sm->tfull1[use & 1u]));
                __syncwarp();
            }
            cluster_wait();                                 // (1)
            cluster_arrive();
            cluster_wait();                                 // (2)
            cluster_arrive();
            cluster_wait();                                 // (3): T of all rows is here, as bf16 terms
            fence_proxy_async_all();
            for (int j = 0; ok && j < nc1 - nc0; ++j, at.advance(1, slots)) {
                const int s = at.slot;
                const unsigned buf = (unsigned)j & 1u;
                ok = warp_wait_spin(smem_u32(&sm->tempty2[buf]), ((used2 >> buf) & 1u) ^ 1u, abort, p.wait.cycles) &&
                     warp_wait_spin(smem_u32(&sm->full[s]), at.round & 1u, abort, p.wait.cycles);
                if (!ok) break;
                used2 ^= 1u << buf;
                tc_fence_after();
                if (elect_one()) {
                    unsigned acc = 0;
#pragma unroll
                    for (int q = C::TERMS - 1; q >= 0; --q) // the smallest term first
#pragma unroll
                        for (int r = 0; r < R / 16; ++r) {
                            const unsigned long long td = make_desc(smem_u32(sT + (q * C::BLOCKS + r / 4) * C::ROWS_BYTES));
                            const unsigned long long bd = make_desc(smem_u32(ring + s * C::SLOT + C::ROWS_BYTES + (r / 4) * C::CW * 128));
                            umma_bf16(tmem_base + 256u + buf * 64u, td + 2ull * (r % 4), bd + 2ull * (r % 4), make_idesc(C::CW), acc);
                            acc = 1;
                        }
                    umma_commit(smem_u32(&sm->tfull2[buf]));
                }
                __syncwarp();
            }
        }
        // everything this thread issued must have retired before tensor memory is freed
        if (elect_one()) umma_commit(smem_u32(&sm->drain));
        __syncwarp();
        mbar_wait(smem_u32(&sm->drain), 0, &sm->drain_abort, p.wait.cycles);
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane, tid = threadIdx.x - 64;
        constexpr int MINE = R >= 64 ? R / 2 : R;           // columns of T a warp takes (up to 32 ranks: the first four warps)
        constexpr int LD = MINE < 32 ? 16 : 32;
        const int col0 = R >= 64 ? half * MINE : 0;
        const bool has_t = R >= 64 || half == 0;
        bool ok = true;
        Place at;                                           // of the chunk in hand (its stages' slots are skipped)
        unsigned use = 0, used2 = 0;
#pragma unroll 1
        for (int it = 0; it < items; ++it) {
            const int row0 = sm->row0[it], count = sm->count[it], a = sm->adapter[it];
            if (a < 0) {
                copy_rows<F32, 8>(p, [&](int r) { return row0 + r; }, count, nc0 * C::CW, min(p.rows, nc1 * C::CW), warp - 2, 8);
                __syncwarp();
                continue;
            }
            cluster_arrive();
            // ---------------- T of this CTA's slice ----------------
            float t[MINE];
#pragma unroll
            for (int j = 0; j < MINE; ++j) t[j] = 0.f;
            for (int k0 = ks0; ok && k0 < ks1; k0 += PIECE, ++use) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm->tfull1[use & 1u]), (use >> 1) & 1u, abort, p.wait.cycles));
                if (!ok) break;
                tc_fence_after();
                if (has_t) {
#pragma unroll
                    for (int q = 0; q < MINE / LD; ++q) {
                        unsigned v[LD];
                        const unsigned at = tmem_base + ((unsigned)(quarter * 32) << 16) + (use & 1u) * R + (unsigned)(col0 + q * LD);
                        if constexpr (LD == 16) tmem_ld_16(at, v);
                        else tmem_ld32(at, v);
#pragma unroll
                        for (int j = 0; j < LD; ++j) t[q * LD + j] += __uint_as_float(v[j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm->tempty1[use & 1u]));
            }
            const float scale = p.scale ? __ldg(p.scale + a) : 1.f;
            // eight ranks of a row, scaled, as bf16 terms, to T of CTAs o0 .. o1 - 1
            auto give = [&](float (&f)[8], int r, int q8, int o0, int o1) {
                const unsigned place = smem_u32(sT) + (unsigned)(q8 / 8) * C::ROWS_BYTES + swz((unsigned)r, (unsigned)q8 & 7u);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = 8 * q8 + j < p.rank ? f[j] * scale : 0.f;   // (as in the kernel for few rows)
#pragma unroll
                for (int q = 0; q < C::TERMS; ++q) {
                    unsigned w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = q + 1 < C::TERMS ? next_terms<false>(f[2 * j], f[2 * j + 1]) : next_terms<true>(f[2 * j], f[2 * j + 1]);
#pragma unroll 1
                    for (int o = o0; o < o1; ++o) {
                        unsigned at;
                        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(place + (unsigned)(q * C::BLOCKS * C::ROWS_BYTES)), "r"(o));
                        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    }
                }
            };
            // To the CTA that adds up this row: [CTA it comes from][four ranks][row], 16 bytes each, rows next to one another.
            const int owner = ((row + 1) * ctas - 1) / 128, most = (128 + ctas - 1) / ctas;
            const unsigned there = smem_u32(sums + (c * (R / 4) + col0 / 4) * most + row - 128 * owner / ctas);
            cluster_wait();                                 // (1)
            if (ctas > 1 && has_t) {
                unsigned at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(there), "r"(owner));
#pragma unroll
                for (int j = 0; j < MINE / 4; ++j)
                    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                                 ::"r"(at + (unsigned)(j * most * 16)), "f"(t[4 * j]), "f"(t[4 * j + 1]), "f"(t[4 * j + 2]), "f"(t[4 * j + 3]) : "memory");
            }
            cluster_arrive();
            cluster_wait();                                 // (2)
            if (ctas == 1) {
                if (has_t) {
#pragma unroll
                    for (int j = 0; j < MINE / 8; ++j) {
                        float f[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = t[8 * j + e];
                        give(f, row, col0 / 8 + j, 0, 1);
                    }
                }
            } else {
                // this CTA's share of the rows: added up and given to all
                const int r0 = 128 * c / ctas, nr = 128 * (c + 1) / ctas - r0;
#pragma unroll 1
                for (int e = tid; e < nr * (R / 8); e += 256) {
                    const int rr = e % nr, q8 = e / nr;
                    float f[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
                        for (int o = 0; o < ctas; ++o) {
                            const float4 v = sums[(o * (R / 4) + 2 * q8 + h) * most + rr];
                            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                        }
                        f[4 * h] = s.x; f[4 * h + 1] = s.y; f[4 * h + 2] = s.z; f[4 * h + 3] = s.w;
                    }
                    give(f, r0 + rr, q8, 0, ctas);
                }
            }
            fence_proxy_async_all();
            __syncwarp();
            cluster_arrive();
            cluster_wait();                                 // (3)
            // ---------------- chunks of Y: four warps take the even ones, four the odd ones ----------------
            const int rows_here = min(32, max(0, count - quarter * 32));
            at.round += (unsigned)(ks1 - ks0) / slots;
            at.advance((ks1 - ks0) % slots + half, slots);
#pragma unroll 1
            for (int j = half; ok && j < nc1 - nc0; j += 2, ++used2, at.advance(2, slots)) {
                const int i = nc0 + j, s = at.slot;
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm->tfull2[half]), used2 & 1u, abort, p.wait.cycles) &&
                                                 mbar_wait(smem_u32(&sm->full[s]), at.round & 1u, abort, p.wait.cycles));
                if (!ok) break;
                tc_fence_after();
                unsigned v[C::CW / 32][32];
                if (rows_here > 0) {
#pragma unroll
                    for (int q = 0; q < C::CW / 32; ++q)
                        tmem_ld32(tmem_base + ((unsigned)(quarter * 32) << 16) + 256u + (unsigned)(half * 64 + q * 32), v[q]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm->tempty2[half]));
                unsigned char *box = ring + s * C::SLOT + quarter * 4096;
                const int n0 = i * C::CW;
                if (rows_here > 0) {
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        uint4 *at = reinterpret_cast<uint4 *>(box + lane * 128 + ((g ^ (lane & 7)) << 4));
                        uint4 y = p.Y0 ? *at : make_uint4(0, 0, 0, 0);
                        if (F32) {
                            y.x = __float_as_uint(__uint_as_float(y.x) + __uint_as_float(v[0][4 * g]));
                            y.y = __float_as_uint(__uint_as_float(y.y) + __uint_as_float(v[0][4 * g + 1]));
                            y.z = __float_as_uint(__uint_as_float(y.z) + __uint_as_float(v[0][4 * g + 2]));
                            y.w = __float_as_uint(__uint_as_float(y.w) + __uint_as_float(v[0][4 * g + 3]));
                        } else {
                            unsigned w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const int e = 8 * g + 2 * q;
                                const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(w[q] << 16) + __uint_as_float(v[e / 32 % (C::CW / 32)][e % 32]),
                                                                               __uint_as_float(w[q] & 0xffff0000u) + __uint_as_float(v[e / 32 % (C::CW / 32)][e % 32 + 1]));
                                w[q] = *reinterpret_cast<const unsigned *>(&h);
                            }
                            y = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        *at = y;
                    }
                    // Whole boxes, clipped at the last column by the map, which clips a store at 16 bytes only.
                    // (The fence is for all ways out: the store, and the slot's next load, come behind what the lanes wrote.)
                    fence_proxy_async();
                    __syncwarp();
                    constexpr int unit = C::CW / 8;
                    const int r0 = lane >> 3, g = lane & 7;
                    const long long first_at = (long long)(row0 + quarter * 32 + r0) * p.ldy + n0 + g * unit;
                    if (rows_here == 32 && (n0 + C::CW <= p.rows || p.rows % unit == 0)) {
                        if (lane == 0) {
                            tma_store_2d(&tm_y, smem_u32(box), n0, row0 + quarter * 32);
                            bulk_commit();
                            bulk_wait_read();                   // (a slot given back a chunk later, unread stores or not: 54 us instead of 50)
                        }
                    } else if (n0 + C::CW <= p.rows) {          // the rows behind are another segment's
                        unsigned char *to = reinterpret_cast<unsigned char *>(p.Y) + first_at * (F32 ? 4 : 2);
#pragma unroll 1
                        for (int b = r0; b < rows_here; b += 8, to += 8 * p.ldy * (F32 ? 4 : 2)) {
                            uint4 y[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                if (b + 4 * i < rows_here) y[i] = *reinterpret_cast<const uint4 *>(box + (b + 4 * i) * 128 + ((g ^ ((b + 4 * i) & 7)) << 4));
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                if (b + 4 * i < rows_here) *reinterpret_cast<uint4 *>(to + 4 * i * p.ldy * (F32 ? 4 : 2)) = y[i];
                        }
                    } else {                                    // and the columns behind are the caller's
                        const int left = p.rows - n0 - g * unit;
                        for (int b = 0; b < rows_here; b += 4) {
                            const int r = b + r0;
                            if (r < rows_here && left > 0) {
                                const uint4 y = *reinterpret_cast<const uint4 *>(box + r * 128 + ((g ^ (r & 7)) << 4));
                                const long long at = first_at + b * p.ldy;
                                if (left >= unit) {
                                    *reinterpret_cast<uint4 *>(reinterpret_cast<unsigned char *>(p.Y) + at * (F32 ? 4 : 2)) = y;
                                } else {
                                    const unsigned w[4] = {y.x, y.y, y.z, y.w};
                                    for (int e = 0; e < left; ++e) {
                                        if (F32) reinterpret_cast<unsigned *>(p.Y)[at + e] = e == 0 ? w[0] : e == 1 ? w[1] : w[2];
                                        else {
                                            const unsigned u = e < 2 ? w[0] : e < 4 ? w[1] : e < 6 ? w[2] : w[3];
                                            reinterpret_cast<unsigned short *>(p.Y)[at + e] = (unsigned short)(e & 1 ? u >> 16 : u);
                                        }
                                    }
                                }
                            }
                        }
                    }
                }
                __syncwarp();                                   // all lanes have read the box before it is given back
                if (lane == 0) mbar_arrive(smem_u32(&sm->empty[s]));
            }
            // on to the first slot behind this item's chunks
            if (half) {
                if ((nc1 - nc0) % 2 == 0) at.retreat(slots);
            } else if ((nc1 - nc0) % 2) at.retreat(slots);
        }
        if (lane == 0) bulk_wait_all();
        __syncwarp();
    }

    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0) {
        if (*abort) atomicOr(p.dev_status, (unsigned)MWU_DEV_TIMEOUT);
        if (total < 0 && blockIdx.x == 0) atomicOr(p.dev_status, (unsigned)MWU_DEV_BOUNDS);
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------
template <int R, bool F32>
static cudaError_t launch_few(const Params &p, int sm_count, cudaStream_t st) {
    auto kern = mwu_adapters_few_kernel<R, F32>;
    const size_t smem = sizeof(Few<R, F32>);
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    // a cluster for every 16 rows that there may be of a segment or an adapter, as far as four CTAs an SM go; more items are taken in turn
    long long items = p.M / 16 + (p.sorted ? p.adapters + 1ll : (long long)p.segments);
    if (!p.sorted && items > 2ll * p.segments) items = 2ll * p.segments;
    if (items > p.M) items = p.M;
    // CTAs to a cluster: as many as leave the SMs with two (of those that are to be expected: half of the adapters in use).  64 rows of 32
    // adapters, 4096 -> 16384, rank 32: 16.6 us with eight, 19.9 with six, 20.4 with four; beside 2777 rows of prompts, 61 rows, 1216 ->
    // 1000: 23.6 with two, 24.4 / 31.1 with four / eight.
    const long long expected = p.sorted ? p.M / 16 + ((p.adapters + 1ll < p.M ? p.adapters + 1ll : p.M) + 1) / 2 : items;
    long long ctas = 7ll * sm_count / (4 * expected);
    ctas = ctas < 2 ? 2 : ctas > 8 ? 8 : ctas;
    const long long most = 4ll * sm_count / ctas;
    count_launch();
    return launch_chained(kern, dim3((unsigned)(ctas * (items < most ? items : most))), dim3(FEW_THREADS), smem, st, (int)ctas, p);
}

static bool encode(CUtensorMap *tm, const void *ptr, bool fp32, int64_t inner, int64_t rows, int64_t ld, int box_rows, int64_t n, int64_t stride) {
    const int64_t size = fp32 ? 4 : 2;
    const cuuint64_t gdim[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)n};
    const cuuint64_t gstride[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(stride * size)};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return get_encode_fn()(tm, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, n ? 3 : 2, const_cast<void *>(ptr),
                           gdim, gstride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// clusters of `ctas` CTAs of the tile kernel that this device runs at a time: a fact of the device, asked once for each
template <int R, bool F32>
static long long clusters_at_once(int ctas, int sm_count) {
    constexpr int DEVICES = 64;
    static std::atomic<int> known[DEVICES][9];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= DEVICES) return sm_count / ctas;
    int n = known[dev][ctas].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = ctas;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(ctas);
        cfg.blockDim = dim3(TILE_THREADS);
        cfg.dynamicSmemBytes = TileCfg<R, F32>::SMEM;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, mwu_adapters_tile_kernel<R, F32>, &cfg) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            n = sm_count / ctas;
        }
        known[dev][ctas].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int R, bool F32>
static int launch_tile(const Params &p, int sm_count, cudaStream_t st) {
    auto kern = mwu_adapters_tile_kernel<R, F32>;
    using C = TileCfg<R, F32>;
    constexpr int smem = C::SMEM;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return MWU_ERR_CUDA;
    if (!get_encode_fn()) return MWU_ERR_CUDA;
    // CTAs of a cluster: what an estimate in microseconds says, of the items that are to be expected (half of the segments that may be long
    // are).  A round takes what it takes to begin and to add up T, and a CTA's share of X, Y0, Y, A and B at 50 GB/s.  Any choice gives every
    // row its adapter.  (8192 rows, 4096 -> 4096, rank 64: two 50 us, four 55; 2777 rows of prompts, 1216 -> 1000, fp32: four 20.2, two
    // 22.5, eight 25.)
    const long long longer = p.M / (FEW_ROWS + 1), some = longer < p.segments ? longer : p.segments;
    const long long expected = (p.M + TILE_ROWS - 1) / TILE_ROWS + (some < p.M / 256 ? some : p.M / 256) / 2;
    const double size = F32 ? 4 : 2;
    const double item = TILE_ROWS * (2.0 * p.cols + (p.Y0 ? 2.0 : 1.0) * size * p.rows) + 2.0 * p.rank * ((double)p.rows + p.cols);
    double best = 1e30;
    int ctas = 1;
    for (int n = 1; n <= 8; ++n) {
        if (C::POW2 && (n & (n - 1))) continue;
        const long long places = clusters_at_once<R, F32>(n, sm_count), rounds = (expected + places - 1) / places;
        const double us = rounds * ((n > 1 ? 6.0 : 4.0) + item / n / 50e3);
        if (us < 0.97 * best) { best = us; ctas = n; }
    }
    const long long most = p.M / TILE_ROWS + some, places = clusters_at_once<R, F32>(ctas, sm_count);
    long long clusters = most < places ? most : places;
    if (clusters < (most + TILE_ITEMS - 1) / TILE_ITEMS) clusters = (most + TILE_ITEMS - 1) / TILE_ITEMS;
    CUtensorMap tm_x, tm_a, tm_b, tm_y0, tm_y;
    if (!encode(&tm_x, p.X, false, p.cols, p.M, p.ldx, 32, 0, 0) || !encode(&tm_a, p.A, false, p.cols, p.rank, p.lda, R, p.adapters, p.a_stride) ||
        !encode(&tm_b, p.B, false, p.rank, p.rows, p.ldb, C::CW, p.adapters, p.b_stride) || !encode(&tm_y, p.Y, F32, p.rows, p.M, p.ldy, 32, 0, 0))
        return MWU_ERR_CUDA;
    tm_y0 = tm_y;                                           // without Y0 it is not used
    if (p.Y0 && p.Y0 != p.Y && !encode(&tm_y0, p.Y0, F32, p.rows, p.M, p.ldy, 32, 0, 0)) return MWU_ERR_CUDA;
    count_launch();
    return launch_chained(kern, dim3((unsigned)(clusters * ctas)), dim3(TILE_THREADS), smem, st, ctas, tm_x, tm_a, tm_b, tm_y0, tm_y, p) ==
                   cudaSuccess ? MWU_OK : MWU_ERR_CUDA;
}

template <int R, bool F32>
static int launch_both(Params p, int sm_count, cudaStream_t st) {
    p.few_rows = 0x7fffffff;
    p.sorted = p.M <= SORTED_ROWS;
    if (p.M > FEW_IN_ALL) {
        p.few_rows = FEW_ROWS;
        const int rc = launch_tile<R, F32>(p, sm_count, st);
        if (rc != MWU_OK) return rc;
        p.beside = 1;
    }
    return launch_few<R, F32>(p, sm_count, st) == cudaSuccess ? MWU_OK : MWU_ERR_CUDA;
}

template <bool F32>
static int launch_rank(const Params &p, int sm_count, cudaStream_t st) {
    if (p.rank <= 16) return launch_both<16, F32>(p, sm_count, st);
    if (p.rank <= 32) return launch_both<32, F32>(p, sm_count, st);
    if (p.rank <= 64) return launch_both<64, F32>(p, sm_count, st);
    return launch_both<128, F32>(p, sm_count, st);
}

}  // namespace adapters
}  // namespace mwu

extern "C" int mwu_adapters_add(int64_t adapters, int64_t rank, int64_t rows, int64_t cols, const void *A, int64_t lda, int64_t a_stride,
                                const void *B, int64_t ldb, int64_t b_stride, const float *scale, int64_t segments,
                                const int32_t *offsets, const int32_t *which, const void *X, int64_t M, int64_t ldx, const void *Y0,
                                void *Y, int64_t ldy, int32_t y_dtype, uint32_t *dev_status, void *cuda_stream) {
    using namespace mwu;
    if (!A || !B || !offsets || !dev_status || M < 0 || (segments > 0 && !which) || (M > 0 && (!X || !Y)))      // (an empty tensor has no address)
        return MWU_ERR_INVALID_ARG;
    if (y_dtype != 0 && y_dtype != 1) return MWU_ERR_INVALID_ARG;
    if (adapters <= 0 || adapters >= (int64_t(1) << 31) || segments < 0 || segments > MWU_MAX_SEGMENTS) return MWU_ERR_SHAPE;
    if (rank <= 0 || rank > MWU_MAX_RANK || rows <= 0 || cols <= 0 || lda < cols || ldb < rank || ldx < cols || ldy < rows) return MWU_ERR_SHAPE;
    if (rows > MWU_MAX_GROUPED_SIDE || cols > MWU_MAX_GROUPED_SIDE || M >= (int64_t(1) << 31) - 256) return MWU_ERR_SHAPE;
    if (lda >= (int64_t(1) << 31) || ldb >= (int64_t(1) << 31) || ldx >= (int64_t(1) << 31) || ldy >= (int64_t(1) << 31)) return MWU_ERR_SHAPE;
    if (a_stride < rank * lda || b_stride < rows * ldb || a_stride >= (int64_t(1) << 38) || b_stride >= (int64_t(1) << 38)) return MWU_ERR_SHAPE;
    if (!aligned_to(A, 16) || !aligned_to(B, 16) || !aligned_to(X, 16) || !aligned_to(Y0, 16) || !aligned_to(Y, 16) || !aligned_to(scale, 4) ||
        !aligned_to(offsets, 4) || !aligned_to(which, 4) || !aligned_to(dev_status, 4) || lda % 8 != 0 || ldb % 8 != 0 || ldx % 8 != 0 ||
        a_stride % 8 != 0 || b_stride % 8 != 0 || ldy % (y_dtype ? 4 : 8) != 0)
        return MWU_ERR_ALIGNMENT;
    int sm_count = 0;
    const int rc = check_device(&sm_count);
    if (rc != MWU_OK) return rc;
    if (M == 0 || segments == 0) return MWU_OK;
    adapters::Params p = {};
    p.A = (const __nv_bfloat16 *)A; p.B = (const __nv_bfloat16 *)B; p.X = (const __nv_bfloat16 *)X;
    p.lda = lda; p.a_stride = a_stride; p.ldb = ldb; p.b_stride = b_stride; p.ldx = ldx; p.ldy = ldy;
    p.scale = scale; p.offsets = offsets; p.which = which; p.Y0 = Y0; p.Y = Y;
    p.adapters = (int)adapters; p.rank = (int)rank; p.rows = (int)rows; p.cols = (int)cols; p.segments = (int)segments; p.M = (int)M;
    p.dev_status = dev_status;
    p.wait = gemm::wait_limits();
    return y_dtype ? adapters::launch_rank<true>(p, sm_count, (cudaStream_t)cuda_stream)
                   : adapters::launch_rank<false>(p, sm_count, (cudaStream_t)cuda_stream);
}
