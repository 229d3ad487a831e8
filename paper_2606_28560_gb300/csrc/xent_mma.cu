// xent_mma.cu -- linear cross entropy on the fifth-generation tensor cores.
//
// Three passes share one engine, a product C[i][j] = sum_k A[i][k] B[j][k] in
// tiles of 256 x 256 over a pair of CTAs (each holds 128 rows of A and half of
// the columns' B; one thread of the even CTA issues the MMAs for both):
//   forward  A = x, B = w, depth D: a row's running maximum and sum of exp
//   gradient A = x, B = w of a piece of the vocabulary: g in bf16 to memory
//   products A = g, B = w (dx, depth: the piece) and A = g^T, B = x (dw, depth N)
// Warp 0 loads (TMA), warp 1 multiplies, warps 4..11 take the accumulators out
// of TMEM: warp w reads lanes 32 (w % 4).. and columns 128 ((w - 4) / 4)... of
// the tile, so a thread owns 128 columns of one row and a row's statistics need
// no exchange.  Two accumulators of 256 columns alternate (or, for products
// wider than 256 columns, are two halves of a tile of 512 that shares A).
//
// The tensor core truncates as it accumulates (for each 16 of depth it loses 2e-8
// of a sum 512 deep, 9e-8 of one 2^15 deep or more, all terms of one sign), so a long
// depth is cut into runs whose sums are added in fp32: 512 deep for bf16 logits,
// whose loss and lse are fp32 results, and 2^15 for the products of bf16 gradients,
// rounded to 8 bits at the end (2^18 rows of positive terms: dw 1.8e-4 low, a tenth
// of such a rounding; 1.3e-3 uncut; at no cost in time).
// fp32 operands are sums of three bf16 planes ("wide" below: several planes,
// runs of 128, CUDA's expf).  The exponentials of bf16 logits are the hardware's exp2:
// with it and the runs of 512, lse and loss of 4096 x 512 x 32768 are 1.9e-7 off their
// values, those of a plain fp32 form 1.1e-7.
#include <algorithm>
#include <atomic>

#include "tc5.cuh"
#include "xent.cuh"
#include "xent_mma.cuh"

namespace fibattn {
namespace xent {
namespace {

constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr unsigned kOperandBytes = 16384;          // 128 rows x 64 deep, bf16
constexpr float kLog2e = 1.4426950408889634f;
// exp(s - m) goes as exp2(s log2e - m log2e) in one FMA.  Beyond this the second term
// may overflow, and the difference is taken first: a tile's row whose tokens are all
// masked by the lowest bf16 value has such an m.
constexpr float kFarLogit = 0x1p126f;
constexpr int kDeepest = 1 << 15;                  // of products of bf16 values: depth that the tensor core sums alone

enum Mode { kForward, kGradient, kProducts };

// RESIDENT: the tile's rows of A stay in shared memory for a unit of tiles (up
// to kResidentChunks chunks of depth), and only B goes through the stages.
constexpr int kResidentChunks = 8;
template <int MODE, int NB, bool RESIDENT> struct Config {
    static constexpr unsigned kResidentBytes = RESIDENT ? kResidentChunks * kOperandBytes : 0;
    static constexpr unsigned kStageBytes = kOperandBytes * ((RESIDENT ? 0 : 1) + NB);
    static constexpr int kStages = RESIDENT ? (MODE == kGradient ? 4 : 6) : NB == 2 ? 4 : MODE == kGradient ? 6 : 7;
    static constexpr unsigned kStoreBytes = MODE == kGradient ? kEpilogueWarps * 4096 : 0;   // a 32 x 64 box a warp
    static constexpr unsigned kSmem = kResidentBytes + kStages * kStageBytes + kStoreBytes + 1024;
};

// One tile (or a part of its depth): rows from m0, columns from n0, depth in
// chunks of 64 from k0 to k1.
struct Item {
    int m0, n0, k0, k1;
    int problem = 0;                               // products: 0 dx, 1 dw
    int unit;                                      // forward, gradient: segment of the columns
    bool first, last;                              // forward, gradient: tile of its unit
    bool whole;                                    // products: the whole depth
    bool begins;                                   // products: the cluster's range begins in this tile
};

// Products: the range of cluster c.  The clusters below first_dw work on dx, the
// others on dw.  Of each product, `siblings` neighbouring clusters take the same
// rows and depth at the same time for different columns, so that what they read
// of g is read from memory once; a sibling's tiles' chunks, one tile after
// another, are cut into equal shares for the groups of siblings.  A boundary
// within `snap` chunks of a tile's end moves there: a sliver is not worth a tile
// of partial sums.
struct Range {
    int problem, sibling, lo, hi;                  // chunks of the sibling's tiles
};
__host__ __device__ inline int share_start(const Product& p, int snap, int group, int groups) {
    const int b = (int)((long long)p.tiles * p.chunks * group / groups), off = b % p.chunks;
    if (off <= snap) return b - off;
    if (p.chunks - off <= snap) return b - off + p.chunks;
    return b;
}
__host__ __device__ inline Range range_of(const Args& a, int c, int clusters) {
    Range r;
    r.problem = c < a.first_dw ? 0 : 1;
    const Product& p = a.prob[r.problem];
    const int local = r.problem ? c - a.first_dw : c, groups = (r.problem ? clusters - a.first_dw : a.first_dw) / p.siblings;
    const int group = local / p.siblings;
    r.sibling = local % p.siblings;
    r.lo = share_start(p, a.snap[r.problem], group, groups);
    r.hi = share_start(p, a.snap[r.problem], group + 1, groups);
    return r;
}
// Tile t of a sibling: its first row and column.
__host__ __device__ inline int tile_row(const Product& p, int t) { return t / (p.col_tiles / p.siblings) * 256; }
__host__ __device__ inline int tile_col(const Args& a, const Product& p, int t, int sibling) {
    return (t % (p.col_tiles / p.siblings) * p.siblings + sibling) * a.tile_cols;
}

// The items of cluster c, in order.
template <int MODE> struct Walk {
    const Args& a;
    int clusters, at, sub;
    Range range;
    __device__ Walk(const Args& args, int cluster, int n) : a(args), clusters(n), at(cluster), sub(0) {
        if (MODE == kProducts) {
            range = range_of(a, cluster, n);
            at = range.lo;
        }
    }
    __device__ bool next(Item& it) {
        if (MODE != kProducts) {
            if (at >= a.units) return false;
            const int mt = at % a.row_tiles, s = at / a.row_tiles;
            const int lo = s * a.unit_tiles, hi = min(a.col_tiles, lo + a.unit_tiles);
            it.m0 = mt * 256;
            it.n0 = (lo + sub) * 256;
            it.k0 = 0;
            it.k1 = a.chunks;
            it.unit = s;
            it.first = sub == 0;
            it.last = lo + sub + 1 >= hi;
            if (it.last) { sub = 0; at += clusters; }
            else ++sub;
            return true;
        } else {
            if (at >= range.hi) return false;
            it.problem = range.problem;
            const Product& p = a.prob[it.problem];
            const int t = at / p.chunks, first = t * p.chunks;
            const int stop = min(range.hi, first + p.chunks);
            it.m0 = tile_row(p, t);
            it.n0 = tile_col(a, p, t, range.sibling);
            it.k0 = at - first;
            it.k1 = stop - first;
            it.whole = it.k0 == 0 && it.k1 == p.chunks;
            it.begins = range.lo >= first;
            at = stop;
            return true;
        }
    }
};

// Columns of block b of a product's tile that are multiplied: a multiple of 32.
__device__ __forceinline__ int block_columns(const Args& a, const Item& it, int b) {
    return min(256, max(0, (min(a.out_cols - it.n0, a.tile_cols) - 256 * b + 31) & ~31));
}

// Boxes of 64 columns that each CTA of the pair loads of them.
__device__ __forceinline__ int block_boxes(const Args& a, const Item& it, int b) { return (block_columns(a, it, b) + 127) / 128; }

// COUNT columns of one output row from registers.  `aligned`: rows start on
// 16-byte boundaries (then no group of 16 bytes straddles the end of a row).
template <int COUNT> __device__ __forceinline__ void put_row(float* out, const float* v, int n, bool aligned) {
    if (aligned) {
#pragma unroll
        for (int j = 0; j < COUNT; j += 4)
            if (j < n) *reinterpret_cast<float4*>(out + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (j < n) out[j] = v[j];
    }
}
template <int COUNT> __device__ __forceinline__ void put_row(__nv_bfloat16* out, const float* v, int n, bool aligned) {
    if (aligned) {
#pragma unroll
        for (int j = 0; j < COUNT; j += 8)
            if (j < n) Vec8<__nv_bfloat16>::store(out + j, v + j);
    } else {
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (j < n) out[j] = __float2bfloat16(v[j]);
    }
}

// Row `row`, n columns (COUNT at most) from c0 of a finished product.  What g was
// divided by is multiplied back here.
template <bool WIDE, int COUNT>
__device__ __forceinline__ void write_product(const Args& a, int problem, int row, int c0, int n, float scale, float* acc) {
    if (row >= a.prob[problem].rows) return;
    const size_t at = (size_t)row * a.out_cols + c0;
    const bool al4 = a.out_cols % 4 == 0;
#pragma unroll
    for (int j = 0; j < COUNT; ++j) acc[j] *= scale;
    if (problem == 0) {
        if (a.dx_add) {
            const float* p = a.dx_acc + at;
            if (al4) {
#pragma unroll
                for (int j = 0; j < COUNT; j += 4)
                    if (j < n) {
                        const float4 v = *reinterpret_cast<const float4*>(p + j);
                        acc[j] += v.x; acc[j + 1] += v.y; acc[j + 2] += v.z; acc[j + 3] += v.w;
                    }
            } else {
#pragma unroll
                for (int j = 0; j < COUNT; ++j)
                    if (j < n) acc[j] += p[j];
            }
        }
        if (!a.dx_done) {
            put_row<COUNT>(a.dx_acc + at, acc, n, al4);
            return;
        }
    }
    void* out = problem == 0 ? a.dx : a.dw;
    const size_t to = problem == 0 ? at : at + (size_t)a.v0 * a.out_cols;
    if (WIDE && a.out_f32) put_row<COUNT>(static_cast<float*>(out) + to, acc, n, al4);
    else put_row<COUNT>(static_cast<__nv_bfloat16*>(out) + to, acc, n, a.out_cols % 8 == 0);
}

// Where a cluster keeps its sums over a part of the depth of a tile: slot 2 c for
// the tile that its range begins in, 2 c + 1 for the one that it ends in.
template <int NB> __device__ __forceinline__ float* slot_at(const Args& a, int slot, int rank, int b, int ew) {
    return a.partials + ((((size_t)slot * 2 + rank) * NB + b) * kEpilogueWarps + ew) * 4096;
}

__device__ __forceinline__ float ex2(float x) { return mma::ex2(x); }
// Two fp32 operations at a time, each rounded as its scalar form.
__device__ __forceinline__ unsigned long long pair(float x, float y) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpair(unsigned long long p, float& x, float& y) {
    asm("mov.b64 {%0, %1}, %2;\n" : "=f"(x), "=f"(y) : "l"(p));
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The largest of 256 threads' values (of 8 warps in a row, t counted from the
// first); they meet at named barrier 1.
__device__ __forceinline__ float block_max(float m, float* red, int t) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (t % 32 == 0) red[t / 32] = m;
    asm volatile("bar.sync 1, 256;\n" ::: "memory");
    m = red[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) m = fmaxf(m, red[w]);
    return m;
}

// g is kept divided by the largest |dloss| of the rows with a target (by 1 if
// there is none or it is not finite): with the mean's equal weights the -1 of a
// target then is exact in bf16, where the weight itself would be off by up to
// 2^-9 in every row alike.  Every block finds it for itself, from all rows or
// from the maxima of another launch.
__device__ __forceinline__ float find_scale(const Args& a, float* red, int t) {
    float m = 0.f;
    if (a.n_maxima > 0) {
        for (int i = t; i < a.n_maxima; i += 256) m = fmaxf(m, a.maxima[i]);
    } else {
        for (int n = t; n < a.p.N; n += 256)
            if (target_column(a.p, n) >= 0) m = fmaxf(m, fabsf(a.dloss[n]));
    }
    m = block_max(m, red, t);
    return m > 0.f && m < INFINITY ? m : 1.f;
}

template <int MODE, int NB, bool WIDE, bool RESIDENT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
xent_kernel(const __grid_constant__ Args a, const __grid_constant__ Maps maps) {
    using C = Config<MODE, NB, RESIDENT>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ unsigned long long bars[2 * C::kStages + 4 + (RESIDENT ? 2 * kResidentChunks : 0)];
    __shared__ unsigned tmem_base_s;
    __shared__ float red_s[MODE == kGradient ? kEpilogueWarps : 1];
    const unsigned smem0 = (tc5::smem_u32(smem_raw) + 1023u) & ~1023u;
    const unsigned full = tc5::smem_u32(bars), empty = full + 8 * C::kStages;
    const unsigned acc_full = empty + 8 * C::kStages, acc_empty = acc_full + 16;
    const unsigned a_full = acc_empty + 16, a_empty = a_full + 8 * kResidentChunks;   // (resident chunks of A)
    const unsigned stages0 = smem0 + C::kResidentBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = tc5::cluster_rank();
    const int cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1;

    if (warp == 0 && lane == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            tc5::init_barrier(full + 8 * s, 1);
            tc5::init_barrier(empty + 8 * s, 1);
        }
        for (int k = 0; RESIDENT && k < kResidentChunks; ++k) {
            tc5::init_barrier(a_full + 8 * k, 1);
            tc5::init_barrier(a_empty + 8 * k, 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc5::init_barrier(acc_full + 8 * b, 1);
            tc5::init_barrier(acc_empty + 8 * b, 2 * kEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        tc5::prefetch_map(&maps.m[0]);
        tc5::prefetch_map(&maps.m[1]);
    }
    if (warp == 2) tc5::tmem_alloc(tc5::smem_u32(&tmem_base_s));
    tc5::fence_before();
    __syncthreads();
    tc5::cluster_sync();
    tc5::fence_after();
    const unsigned tmem = tmem_base_s;
    grid_dependency_sync();
    asm volatile("fence.proxy.async.global;\n" ::: "memory");   // operands written by the kernel before are read by TMA

    const int combos = WIDE ? a.combos : 1;        // products of planes for one of values
    // Depth of a run (chunks of 64) whose sums stay in the tensor core.
    constexpr int kRun = WIDE ? 2 : MODE != kProducts ? 8 : kDeepest / 64;

    if (warp < 4) {
        tc5::registers_down<56>();
        if (warp == 0 && tc5::elect_one()) {
            // ---- loads: this CTA's operands; the even CTA's barrier counts both's bytes
            const unsigned full0 = tc5::map_to(full, 0);
            // x and w are read by every cluster; g passes through once in each product (its
            // planes, where it has several, are read again).  With these hints and 16384
            // rows, 512 wide, 32768 columns: gradient 360 -> 344 us, products 644 -> 614.
            const unsigned long long keep = tc5::policy_keep(), pass = WIDE ? tc5::policy_normal() : tc5::policy_pass();
            Walk<MODE> walk(a, cluster, clusters);
            Item it;
            const unsigned a_full0 = tc5::map_to(a_full, 0);
            int stage = 0;
            unsigned phase = 0, unit = 0;
            int a_upto = 0;                                // chunks of the current unit's rows that are issued
            long long issued = 0;
            bool ok = true;
            while (ok && walk.next(it)) {
                // Bytes of a stage, both CTAs.  Half tiles without a row or a column are not
                // loaded: what a stale operand gives goes to rows and columns that nobody
                // looks at, and boxes that lie outside their tensor are slow to fill.
                const bool a_here = it.problem == 1 || it.m0 + 128 * (int)rank < a.p.N;
                const bool b_here = MODE == kProducts || a.v0 + it.n0 + 128 * (int)rank < a.p.V;
                const unsigned a_bytes = MODE == kProducts && it.problem == 1 ? 2 * kOperandBytes
                                                                              : a.row_box * 128u * (it.m0 + 128 < a.p.N ? 2 : 1);
                unsigned bytes = RESIDENT ? 0 : a_bytes;
                if (MODE != kProducts) {
                    bytes += kOperandBytes * (a.v0 + it.n0 + 128 < a.p.V ? 2 : 1);
                } else {
#pragma unroll
                    for (int b = 0; b < NB; ++b) bytes += 2 * 8192u * block_boxes(a, it, b);
                }
                for (int r0 = it.k0; ok && r0 < it.k1; r0 += min(kRun, it.k1 - r0)) {
                    const int len = min(kRun, it.k1 - r0);
                    for (int i = 0; i < combos * len; ++i) {
                        const int chunk = r0 + (WIDE ? i % len : i);
                        const int pa = WIDE ? (a.combo_a >> (4 * (i / len))) & 15 : 0;
                        const int pb = WIDE ? (a.combo_b >> (4 * (i / len))) & 15 : 0;
                        if (RESIDENT && it.first) {        // the unit's rows, as the last unit's are done with
                            a_upto = chunk;
                            ok = tc5::wait_parity(a_empty + 8 * chunk, (unit & 1u) ^ 1u);
                            if (!ok) break;
                            if (rank == 0) tc5::expect_bytes(a_full + 8 * chunk, a_bytes);
                            if (a_here)
                                tc5::load_box(smem0 + chunk * kOperandBytes, &maps.m[0], chunk * 64, it.m0 + 128 * rank, 0,
                                              a_full0 + 8 * chunk, keep);
                            a_upto = chunk + 1;
                        }
                        ok = tc5::wait_parity(empty + 8 * stage, phase ^ 1u);
                        if (!ok) break;
                        if (rank == 0) tc5::expect_bytes(full + 8 * stage, bytes);
                        const unsigned bar = full0 + 8 * stage, dst = stages0 + stage * C::kStageBytes;
                        if (MODE != kProducts) {
                            if (!RESIDENT && a_here) tc5::load_box(dst, &maps.m[0], chunk * 64, it.m0 + 128 * rank, pa, bar, keep);
                            if (b_here)
                                tc5::load_box(dst + (RESIDENT ? 0 : kOperandBytes), &maps.m[1], chunk * 64,
                                              a.v0 + it.n0 + 128 * rank, pb, bar, keep);
                        } else {
                            if (it.problem == 0) {
                                if (a_here) tc5::load_box(dst, &maps.m[0], chunk * 64, it.m0 + 128 * rank, pa, bar, pass);
                            } else {
                                for (int h = 0; h < 2; ++h)
                                    tc5::load_box(dst + 8192 * h, &maps.m[2], it.m0 + 128 * rank + 64 * h, chunk * 64, pa, bar, pass);
                            }
                            for (int b = 0; b < NB; ++b) {
                                const int n = it.n0 + 256 * b + (int)rank * (block_columns(a, it, b) / 2);
                                // the innermost coordinate starts on a 16-byte boundary: block_columns / 2 is a multiple of 16
                                for (int h = 0; h < block_boxes(a, it, b); ++h)
                                    tc5::load_box(dst + kOperandBytes * (1 + b) + 8192 * h, &maps.m[it.problem == 0 ? 1 : 3],
                                                  n + 64 * h, (it.problem == 0 ? a.v0 : 0) + chunk * 64, pb, bar, keep);
                            }
                        }
                        ++issued;
                        if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                    }
                }
                if (RESIDENT && it.last) {
                    ++unit;
                    a_upto = 0;
                }
            }
            if (!ok) {
                // Copies may still be under way into this pair's shared memory: wait
                // for the stages issued last (bounded as every wait is).
                raise_status(a.p.status, kStatusWaitTimeout);
                if (RESIDENT && rank == 0)
                    for (int k = 0; k < a.chunks; ++k)
                        if (k < a_upto || unit > 0) tc5::wait_parity(a_full + 8 * k, k < a_upto ? unit & 1u : (unit - 1) & 1u);
                if (rank == 0)
                    for (int s = 0; s < C::kStages && s < issued; ++s) {
                        const int st = (stage + C::kStages - 1 - s) % C::kStages;
                        tc5::wait_parity(full + 8 * st, st < stage ? phase : phase ^ 1u);
                    }
            }
        } else if (warp == 1 && rank == 0 && tc5::elect_one()) {
            // ---- multiplications
            Walk<MODE> walk(a, cluster, clusters);
            Item it;
            int stage = 0;
            unsigned phase = 0, run = 0, unit = 0;
            bool ok = true;
            while (ok && walk.next(it)) {
                const bool a_rows = MODE == kProducts && it.problem == 1, b_rows = MODE == kProducts;
                unsigned idesc[NB];
                int cols[NB];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    cols[b] = MODE == kProducts ? block_columns(a, it, b) : 256;
                    idesc[b] = tc5::instruction(cols[b], a_rows, b_rows);
                }
                const int depth = MODE != kProducts ? a.p.D : it.problem == 0 ? a.cols : a.p.N;
                const unsigned a_step = a_rows ? 128u : 2u, b_step = b_rows ? 128u : 2u;   // 16 of depth, in 16 bytes
                for (int r0 = it.k0; ok && r0 < it.k1; r0 += min(kRun, it.k1 - r0), ++run) {
                    const int len = min(kRun, it.k1 - r0);
                    const unsigned buf = NB == 2 ? 0u : run & 1u, use = NB == 2 ? run : run >> 1;
#pragma unroll
                    for (int b = 0; b < NB; ++b) ok = ok && tc5::wait_parity(acc_empty + 8 * (buf + b), (use & 1u) ^ 1u);
                    if (!ok) break;
                    tc5::fence_after();
                    for (int i = 0; i < combos * len; ++i) {
                        if (RESIDENT && it.first) {
                            ok = tc5::wait_parity(a_full + 8 * i, unit & 1u);
                            if (!ok) break;
                        }
                        ok = tc5::wait_parity(full + 8 * stage, phase);
                        if (!ok) break;
                        tc5::fence_after();
                        const int left = depth - 64 * (r0 + (WIDE ? i % len : i));   // what is past the depth is zeros
                        const unsigned src = stages0 + stage * C::kStageBytes;
                        const unsigned long long da = tc5::descriptor(RESIDENT ? smem0 + i * kOperandBytes : src, a_rows ? 8192u : 16u);
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            const unsigned long long db =
                                tc5::descriptor(src + kOperandBytes * ((RESIDENT ? 0 : 1) + b), b_rows ? 8192u : 16u);
                            if (cols[b] > 0) {
#pragma unroll
                                for (unsigned k = 0; k < 4; ++k)
                                    if ((int)(16 * k) < left)
                                        tc5::multiply(tmem + 256 * (buf + b), da + a_step * k, db + b_step * k, idesc[b], i > 0 || k > 0);
                            }
                        }
                        tc5::commit_pair(empty + 8 * stage);
                        if (RESIDENT && it.last) tc5::commit_pair(a_empty + 8 * i);
                        if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
#pragma unroll
                    for (int b = 0; b < NB; ++b) tc5::commit_pair(acc_full + 8 * (buf + b));
                }
                if (RESIDENT && it.last) ++unit;
            }
            if (!ok) raise_status(a.p.status, kStatusWaitTimeout);
        }
    } else {
        tc5::registers_up<224>();
        // ---- epilogue: 128 columns of one row per thread
        const int ew = warp - 4, half = ew >> 2;
        const int lane_row = (warp & 3) * 32 + lane;
        const unsigned t_lane = tmem + ((unsigned)(warp & 3) << 21) + 128u * half;
        const unsigned acc_empty0 = tc5::map_to(acc_empty, 0);
        const unsigned stage_out = stages0 + C::kStages * C::kStageBytes + ew * 4096u;
        Walk<MODE> walk(a, cluster, clusters);
        Item it;
        unsigned run = 0;
        bool ok = true;
        float m = -INFINITY, l = 0.f, z = 0.f, dl = 0.f;
        int target = kIgnored;
        float out_scale = 1.f;
        if (MODE == kGradient) {
            out_scale = find_scale(a, red_s, threadIdx.x - 128);
            if (blockIdx.x == 0 && threadIdx.x == 128) *a.scale = out_scale;
        } else if (MODE == kProducts) {
            out_scale = *a.scale;
        }
        while (walk.next(it)) {
            const int row = it.m0 + 128 * (int)rank + lane_row;
            if (MODE == kForward && it.first) {
                m = -INFINITY;
                l = 0.f;
                target = row < a.p.N ? target_column(a.p, row) : kIgnored;
            }
            if (MODE == kGradient && it.first) {
                target = row < a.p.N ? target_column(a.p, row) : kIgnored;
                z = row < a.p.N ? a.lse[row] : 0.f;
                dl = row < a.p.N ? a.dloss[row] / out_scale : 0.f;
                if (target == kBad && a.v0 + it.n0 == 0 && half == 0) raise_status(a.p.status, kStatusTarget);
            }
            float acc[128];
            const int runs = (it.k1 - it.k0 + kRun - 1) / kRun;
            // A thread has registers for one block's sums: with two blocks the runs of a
            // tile are added up in memory, a turn over the blocks for each run.
            const int turns = NB == 2 ? runs : 1;
#pragma unroll 1
            for (int turn = 0, b = 0; turn < turns; turn += b == NB - 1, b = (b + 1) % NB) {
                unsigned n_run = run;
#pragma unroll 1
                for (int r = 0; r < (NB == 2 ? 1 : runs); ++r, ++n_run) {
                    const unsigned buf = NB == 2 ? (unsigned)b : n_run & 1u, use = NB == 2 ? n_run : n_run >> 1;
                    ok = ok && tc5::wait_parity(acc_full + 8 * buf, use & 1u);
                    if (!ok) continue;
                    tc5::fence_after();
                    const unsigned t = t_lane + 256u * buf;
                    if (r == 0) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) tc5::tmem_load32(t + 32 * q, acc + 32 * q);
                        tc5::tmem_wait_loads();
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float v[32];
                            tc5::tmem_load32(t + 32 * q, v);
                            tc5::tmem_wait_loads();
#pragma unroll
                            for (int j = 0; j < 32; ++j) acc[32 * q + j] += v[j];
                        }
                    }
                    tc5::fence_before();
                    __syncwarp();
                    if (lane == 0) tc5::arrive_cluster(acc_empty0 + 8 * buf);
                }
                if (b == NB - 1) run = n_run;
                if (!ok) {                          // the accumulators never came: every output of this tile is NaN
                    if (lane == 0) raise_status(a.p.status, kStatusWaitTimeout);
#pragma unroll
                    for (int j = 0; j < 128; ++j) acc[j] = NAN;
                }
                const int c0 = it.n0 + 256 * b + 128 * half;

                if (MODE == kForward) {
                    if (c0 + 128 > a.p.V) {
#pragma unroll
                        for (int j = 0; j < 128; ++j)
                            if (c0 + j >= a.p.V) acc[j] = -INFINITY;
                    }
                    if ((unsigned)(target - c0) < 128u) {
                        float s = 0.f;
#pragma unroll
                        for (int j = 0; j < 128; ++j) s = c0 + j == target ? acc[j] : s;
                        a.parts.target_logit[row] = s;
                    }
                    float mx[4] = {m, acc[0], acc[1], acc[2]};
#pragma unroll
                    for (int j = 3; j < 127; j += 2) mx[j / 2 & 3] = max3(mx[j / 2 & 3], acc[j], acc[j + 1]);
                    const float top = max3(max3(mx[0], mx[1], mx[2]), mx[3], acc[127]);
                    const float ms = top == -INFINITY ? 0.f : top;
                    float s[4] = {0.f, 0.f, 0.f, 0.f};
                    if (WIDE) {
#pragma unroll
                        for (int j = 0; j < 128; ++j) s[j & 3] += expf(acc[j] - ms);
                        l = l * expf(m - ms);
                    } else {
                        float off = -ms * kLog2e;
                        if (fabsf(ms) > kFarLogit) {
#pragma unroll
                            for (int j = 0; j < 128; ++j) acc[j] -= ms;
                            m -= ms;
                            off = 0.f;
                        }
                        const unsigned long long scale2 = pair(kLog2e, kLog2e), off2 = pair(off, off);
                        unsigned long long s2[2] = {0ull, 0ull};
#pragma unroll
                        for (int j = 0; j < 128; j += 2) {
                            float u, v;
                            unpair(fma2(pair(acc[j], acc[j + 1]), scale2, off2), u, v);
                            s2[j / 2 & 1] = add2(s2[j / 2 & 1], pair(ex2(u), ex2(v)));
                        }
                        unpair(s2[0], s[0], s[1]);
                        unpair(s2[1], s[2], s[3]);
                        l = l * ex2(fmaf(m, kLog2e, off));
                    }
                    l += (s[0] + s[1]) + (s[2] + s[3]);
                    m = top;
                    if (it.last && row < a.p.N) {
                        const size_t at = (size_t)(2 * it.unit + half) * a.p.N + row;
                        a.parts.m[at] = m;
                        a.parts.l[at] = l;
                    }
                } else if (MODE == kGradient) {
                    // a row without a target gives exact zeros, whatever its logits
                    if (target < 0) {
#pragma unroll
                        for (int j = 0; j < 128; ++j) acc[j] = ok ? 0.f : NAN;
                    } else {
                        if (WIDE) {
#pragma unroll
                            for (int j = 0; j < 128; ++j) acc[j] = dl * expf(acc[j] - z);
                        } else {
                            float off = -z * kLog2e;
                            if (fabsf(z) > kFarLogit) {
#pragma unroll
                                for (int j = 0; j < 128; ++j) acc[j] -= z;
                                off = 0.f;
                            }
                            const unsigned long long scale2 = pair(kLog2e, kLog2e), off2 = pair(off, off), dl2 = pair(dl, dl);
#pragma unroll
                            for (int j = 0; j < 128; j += 2) {
                                float u, v;
                                unpair(fma2(pair(acc[j], acc[j + 1]), scale2, off2), u, v);
                                unpair(mul2(pair(ex2(u), ex2(v)), dl2), acc[j], acc[j + 1]);
                            }
                        }
                        const int local = target - a.v0 - c0;
                        if ((unsigned)local < 128u) {
#pragma unroll
                            for (int j = 0; j < 128; ++j)
                                if (j == local) acc[j] -= dl;
                        }
                    }
                    const int r0 = it.m0 + 128 * (int)rank + (warp & 3) * 32;
#pragma unroll
                    for (int plane = 0; plane < (WIDE ? 3 : 1); ++plane) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int col = c0 + 64 * h;
                            if (r0 < a.p.N && col < a.cols) {        // (uniform over the warp)
                                const unsigned dst = stage_out;
                                if (lane == 0) tc5::store_wait_read<0>();
                                __syncwarp();
#pragma unroll
                                for (int ch = 0; ch < 8; ++ch) {
                                    unsigned u[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const int j = 64 * h + 8 * ch + 2 * e;
                                        u[e] = mma::pack_bf16(acc[j], acc[j + 1]);
                                        if (WIDE) {           // what the next plane has to hold
                                            acc[j] -= __uint_as_float(u[e] << 16);
                                            acc[j + 1] -= __uint_as_float(u[e] & 0xffff0000u);
                                        }
                                    }
                                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n"
                                                 :: "r"(mma::row_chunk(dst, lane, ch)), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3])
                                                 : "memory");
                                }
                                tc5::fence_async_smem();
                                __syncwarp();
                                if (lane == 0) {
                                    tc5::store_box(&maps.m[2], dst, col, r0, plane);
                                    tc5::store_commit();
                                }
                            }
                        }
                    }
                } else if constexpr (MODE == kProducts) {
                    const int end = min(a.out_cols, it.n0 + a.tile_cols);
                    if (c0 >= end) continue;                 // (uniform over the warp)
                    float* mine = slot_at<NB>(a, 2 * cluster + (it.begins ? 0 : 1), (int)rank, b, ew) + lane;
                    const bool in = row < a.prob[it.problem].rows;
                    if (NB == 2 && turn > 0 && in) {         // the runs before, this thread's own
#pragma unroll
                        for (int j = 0; j < 128; ++j) acc[j] += __ldcg(mine + 32 * j);
                    }
                    if (it.whole && turn == turns - 1) {
                        write_product<WIDE, 128>(a, it.problem, row, c0, end - c0, out_scale, acc);
                    } else if (in) {
#pragma unroll
                        for (int j = 0; j < 128; ++j) __stcg(mine + 32 * j, acc[j]);
                    }
                }
            }
        }
        if (MODE == kGradient && lane == 0) tc5::store_wait_all();
    }
    // Neither CTA leaves, or gives up its TMEM, while the other may still use it.
    tc5::fence_before();
    __syncwarp();
    tc5::cluster_sync();
    tc5::fence_after();
    if (warp == 2) tc5::tmem_free(tmem);
}

// maxima[block] = the largest |dloss| of the block's rows that have a target.
__global__ void __launch_bounds__(256) maxima_kernel(Problem p, const float* dloss, float* maxima) {
    __shared__ float red[8];
    grid_dependency_sync();
    float m = 0.f;
    for (int n = blockIdx.x * 256 + threadIdx.x; n < p.N; n += gridDim.x * 256)
        if (target_column(p, n) >= 0) m = fmaxf(m, fabsf(dloss[n]));
    m = block_max(m, red, threadIdx.x);
    if (threadIdx.x == 0) maxima[blockIdx.x] = m;
}

// x, or bf16's largest value with its sign where x is larger; NaN stays.  The planes
// but the last hold this: the lowest fp32 value, a usual mask, would else round to an
// infinity in the first, and an infinity leave NaN in the next.
__device__ __forceinline__ float within_bf16(float x) {
    float r;
    asm("min.NaN.xorsign.abs.f32 %0, %1, %2;\n" : "=f"(r) : "f"(x), "f"(__uint_as_float(0x7f7f0000u)));
    return r;
}

// Rows of T as `planes` bf16 planes of row length `depth`, a multiple of eight
// (zeros past D): one plane rounds nothing (bf16 rows of a length that TMA
// cannot address), three hold an fp32 value to 24 bits.  A thread takes eight
// values; two operands go in one launch.
struct PackJob {
    const void* src;
    __nv_bfloat16* dst;
    long long rows, groups;                        // groups of eight
};
template <typename T> __global__ void __launch_bounds__(256) pack_kernel(PackJob a, PackJob b, int D, int depth, int planes) {
    grid_dependency_sync();
    const int per_row = depth / 8;
    const bool vectors = D % 8 == 0;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < a.groups + b.groups; i += gridDim.x * 256ll) {
        const PackJob& job = i < a.groups ? a : b;
        const long long g = i < a.groups ? i : i - a.groups, r = g / per_row;
        const int c = (int)(g - r * per_row) * 8;
        const T* src = static_cast<const T*>(job.src) + r * D + c;
        float x[8];
        if (vectors && c < D) {                   // (then the whole group is: D is a multiple of eight)
            Vec8<T>::load(src, x);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = c + j < D ? to_f(src[j]) : 0.f;
        }
        for (int p = 0; p < planes; ++p) {
            const bool more = p + 1 < planes;
            unsigned u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u[j] = mma::pack_bf16(more ? within_bf16(x[2 * j]) : x[2 * j], more ? within_bf16(x[2 * j + 1]) : x[2 * j + 1]);
                x[2 * j] -= __uint_as_float(u[j] << 16);
                x[2 * j + 1] -= __uint_as_float(u[j] & 0xffff0000u);
            }
            reinterpret_cast<uint4*>(job.dst)[p * job.groups + g] = make_uint4(u[0], u[1], u[2], u[3]);
        }
    }
}

// x and w as planes at x_to and w_to.
cudaError_t pack(const Problem& p, int depth, int planes, void* x_to, void* w_to, bool bf16, cudaStream_t st) {
    const PackJob x{p.x, static_cast<__nv_bfloat16*>(x_to), p.N, (long long)p.N * (depth / 8)};
    const PackJob w{p.w, static_cast<__nv_bfloat16*>(w_to), p.V, (long long)p.V * (depth / 8)};
    const dim3 grid((unsigned)std::max(1ll, std::min((x.groups + w.groups) / 256 + 1, 152ll * 8)));
    return bf16 ? launch_kernel(pack_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, x, w, p.D, depth, planes)
                : launch_kernel(pack_kernel<float>, grid, dim3(256), 0, st, x, w, p.D, depth, planes);
}

// The tiles that several clusters share: the sums of their parts, in the order
// of the depth, by all SMs.  (A warp that finds itself the last of a tile's parts
// could add them up inside the products; it then reads them through one SM: with
// 64 rows, 512 wide, 32768 columns, where dx is one tile over 24 clusters, that
// took 149 us of products against 26.5 and 8 for this kernel, and with 16384 rows,
// two parts to a tile, the same time.)  Block (tile, group of 32 rows x 128
// columns); a thread takes eight columns of a row.
struct SplitTile {
    int problem, m0, n0, first, parts;             // slots[first ..] hold its parts
};
struct SplitTiles {
    int count;
    SplitTile tile[kClusters];
    short slots[2 * kClusters];
};
template <int NB, bool WIDE>
__global__ void __launch_bounds__(512) join_products_kernel(const __grid_constant__ Args a, const __grid_constant__ SplitTiles s) {
    grid_dependency_sync();
    const SplitTile& t = s.tile[blockIdx.x];
    const int ew = blockIdx.y % kEpilogueWarps, b = blockIdx.y / kEpilogueWarps % NB, rank = blockIdx.y / (kEpilogueWarps * NB);
    const int lane = threadIdx.x & 31, j0 = (threadIdx.x >> 5) * 8;
    const int row = t.m0 + 128 * rank + 32 * (ew & 3) + lane, c0 = t.n0 + 256 * b + 128 * (ew >> 2) + j0;
    const int end = min(a.out_cols, t.n0 + a.tile_cols);
    if (row >= a.prob[t.problem].rows || c0 >= end) return;
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
#pragma unroll 4
    for (int i = 0; i < t.parts; ++i) {
        const float* p = slot_at<NB>(a, s.slots[t.first + i], rank, b, ew) + 32 * j0 + lane;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += __ldcg(p + 32 * j);
    }
    write_product<WIDE, 8>(a, t.problem, row, c0, end - c0, *a.scale, acc);
}

// Which tiles the ranges of `clusters` clusters cut, and where their parts are.
void find_splits(const Args& a, int clusters, SplitTiles* s) {
    s->count = 0;
    int used = 0;
    for (int first = 0; first < clusters; ) {      // the first cluster of a group of siblings
        const Range r = range_of(a, first, clusters);
        const Product& p = a.prob[r.problem];
        const int past = r.problem ? clusters : a.first_dw;
        const int t = r.hi / p.chunks, lo = t * p.chunks;
        if (r.lo <= lo && lo < r.hi) {             // the range holds the first part of tile t, not the last

            for (int sib = 0; sib < p.siblings; ++sib) {
                SplitTile& tile = s->tile[s->count++];
                tile = SplitTile{r.problem, tile_row(p, t), tile_col(a, p, t, sib), used, 0};
                for (int c = first + sib; c < past; c += p.siblings) {
                    const Range part = range_of(a, c, clusters);
                    if (part.lo >= lo + p.chunks) break;
                    if (part.hi <= part.lo || part.hi <= lo) continue;
                    s->slots[used++] = (short)(2 * c + (part.lo >= lo ? 0 : 1));
                    ++tile.parts;
                }
            }
        }
        first += p.siblings;
    }
}

bool encode(CUtensorMap* map, const void* base, long long cols, long long rows, int planes, long long row_len, int box_cols,
            int box_rows) {
    auto fn = tensor_map_encoder();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    cuuint64_t strides[2] = {(cuuint64_t)row_len * 2, (cuuint64_t)(rows * row_len) * 2};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, int NB, bool WIDE, bool RESIDENT>
cudaError_t launch(const Args& a, const Maps& maps, int clusters, cudaStream_t st) {
    auto kern = xent_kernel<MODE, NB, WIDE, RESIDENT>;
    // The register split of the two halves of a block draws on what the block
    // was launched with: refuse to launch a build that was given less.
    static const int registers = [&] {
        cudaFuncAttributes at{};
        return cudaFuncGetAttributes(&at, kern) == cudaSuccess ? at.numRegs : 0;
    }();
    if (registers * kThreads < 56 * 128 + 224 * 256) return cudaErrorInvalidDeviceFunction;
    constexpr unsigned smem = Config<MODE, NB, RESIDENT>::kSmem;
    static std::atomic<unsigned long long> set{0};          // devices (of the first 64) where the limit is raised already
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(set.load(std::memory_order_relaxed) >> dev & 1)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) set.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    return launch_kernel(kern, dim3(2 * clusters), dim3(kThreads), smem, st, a, maps);
}

// Rows of the boxes that x (and g, for dx) are loaded in: whole groups of eight.
int row_box_of(int N) { return std::min(128, (N + 7) / 8 * 8); }

int tiles256(long long n) { return (int)((n + 255) / 256); }
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Whether the rows of a tile stay in shared memory over the tiles of a unit,
// which halves what the forward and the gradient pass load.  16384 rows, 512 wide,
// 32768 columns: the forward 273 -> 261 us; the gradient pass, whose stages then
// are four instead of six, 340 -> 365 us by itself, but the card runs at its power
// limit after some tens of milliseconds and then the step takes 1440 -> 1409 us
// with both, 1420 us with the forward alone.
bool resident(const Args& a) { return a.chunks <= kResidentChunks && a.unit_tiles > 1; }

// Whether the operands are packed, into how many planes and rows of what
// length.  bf16 rows are taken where they lie if TMA can address them (16-byte
// rows); of those, rows that do not start on 32-byte boundaries cost the loads a
// third of their rate, which from some 2500 rows on is more than the packing
// takes (712 wide, 20000 columns, us forward in place / packed: 2048 rows 49.2 /
// 50.4, 4096 rows 88.9 / 81.6, 8192 rows 165 / 147).
void plan_operands(int N, int D, bool bf16, bool* pack, int* planes, int* depth) {
    *pack = !bf16 || D % 8 != 0 || (D % 16 != 0 && N >= 2560);
    *planes = bf16 ? 1 : 3;
    *depth = *pack ? (D + 15) / 16 * 16 : D;
}

// The products of planes that make up one of values, the small ones first:
// while the running sum is small so is what truncation takes from it.  Of the
// nine products of three planes with three, six are kept (the others are below
// 2^-24 of the value).
void set_combos(Args* a, int planes_a, int planes_b) {
    if (planes_a == 3 && planes_b == 3) {
        a->combos = 6;
        a->combo_a = 0x010120;                     // read from the right: 0 2 1 0 1 0
        a->combo_b = 0x001102;                     //                      2 0 1 1 0 0
    } else if (planes_a == 3) {
        a->combos = 3;
        a->combo_a = 0x012;
        a->combo_b = 0;
    } else {
        a->combos = 1;
        a->combo_a = a->combo_b = 0;
    }
}

}  // namespace

// Tiles of one row of tiles that a cluster takes one after another (a unit):
// the fewest rounds over the clusters win, with a quarter of a tile for what a
// unit costs by itself (its rows' targets, the statistics it writes).  At most
// 64 segments of the columns, so that the forward's statistics stay small.
static int unit_tiles_of(int row_tiles, int col_tiles) {
    const int least = std::max(1, (col_tiles + 63) / 64);
    int unit = least;
    double best = 0;
    for (int u = least; u <= std::max(16, least); ++u) {
        const long long units = (long long)row_tiles * ((col_tiles + u - 1) / u);
        const double cost = (double)((units + kClusters - 1) / kClusters) * (u + 0.25);
        if (u == least || cost < best) {
            best = cost;
            unit = u;
        }
    }
    return unit;
}

// Whether products are made of several products of planes.  One bf16 plane rounds
// each g to 8 bits, which the sums of dx and dw average out over many; fp32 I/O
// keeps three planes (24 bits), and so does bf16 I/O where whole tiles come to at
// most 2^26 multiplications: there the sums are short and the further planes hide
// behind the launches (100 rows, 64 wide, 257 columns: 27 us either way).
static bool several_planes(int N, int D, int V, bool bf16) {
    return !bf16 || 256.0 * tiles256(N) * 256.0 * tiles256(V) * D <= (double)(1 << 26);
}

// Forward and backward go the same way: p = exp(logit - lse) is good to the
// logits' own rounding only if both come from the same arithmetic.  Of the three a
// call takes the one that is faster.  Forward and backward together, us on the GPU,
// few rows / tiles:
//                              bf16: 8 rows     16 rows     32 rows    fp32: 32 rows
//   512 wide, 32768 columns:       42 / 67     51 / 67     83 / 62       119 / 203
//   1000 wide, 20000 columns:      52 / 67     63 / 67    102 / 65       154 / 279
//   2048 wide, 131072 columns:   449 / 496   552 / 498   954 / 500     1400 / 2642
//   512 wide, 4000 columns:        21 / 31     24 / 31     27 / 30        39 / 75
//   8192 wide, 20000 columns:    322 / 355                              1475 / 1918
// and stream / few rows:
//                              bf16: 1 row      2 rows      4 rows     fp32: 4 rows
//   512 wide, 32768 columns:       33 / 43     38 / 43     48 / 41        67 / 62
//   1000 wide, 20000 columns:      42 / 51     50 / 51     65 / 51        91 / 81
//   2048 wide, 131072 columns:   372 / 455   425 / 457   517 / 450      802 / 780
//   512 wide, 4000 columns:        13 / 21     14 / 21     17 / 21        18 / 25
static Way way_of(int N, int D, int V, bool bf16) {
    const bool small = (long long)V * D <= (1 << 22);
    if (stream_applies(N, D) && (N <= 2 || small)) return Way::kStream;
    const int most = !bf16 || small ? 32 : D <= 1024 ? 16 : 8;
    return N <= most && few_rows_applies(N) ? Way::kFewRows : Way::kTiles;
}

FwdPlan plan_forward(int N, int D, int V, bool bf16) {
    FwdPlan f{};
    f.way = way_of(N, D, V, bf16);
    if (f.way == Way::kStream) {
        f.segments = stream_segments(V);
    } else if (f.way == Way::kFewRows) {
        f.segments = few_rows_segments(N, D, V);
    } else {
        plan_operands(N, D, bf16, &f.pack, &f.planes, &f.depth);
        f.wide = several_planes(N, D, V, bf16);
        f.unit_tiles = unit_tiles_of(tiles256(N), tiles256(V));
        f.segments = 2 * ((tiles256(V) + f.unit_tiles - 1) / f.unit_tiles);
    }
    size_t off = 0;
    const auto take = [&](size_t n) { const size_t at = off; off += up256(n); return at; };
    f.x = take(f.pack ? (size_t)f.planes * N * f.depth * 2 : 0);
    f.w = take(f.pack ? (size_t)f.planes * V * f.depth * 2 : 0);
    f.m = take((size_t)f.segments * N * 4);
    f.l = take((size_t)f.segments * N * 4);
    f.target = take((size_t)N * 4);
    f.total = off;
    return f;
}

cudaError_t run_forward(const Problem& p, const FwdPlan& f, char* ws, bool bf16, float* loss, float* lse, cudaStream_t st) {
    const FwdParts parts{reinterpret_cast<float*>(ws + f.m), reinterpret_cast<float*>(ws + f.l),
                         reinterpret_cast<float*>(ws + f.target)};
    cudaError_t e;
    if (f.way != Way::kTiles) {
        {
            ProfScope s(f.way == Way::kStream ? "xent_stream" : "xent_few_rows", st);
            e = f.way == Way::kStream ? launch_stream(p, parts, f.segments, bf16, st) : launch_few_rows(p, parts, f.segments, bf16, st);
        }
        if (e != cudaSuccess) return e;
        ProfScope s("xent_join", st);
        return launch_join_rows(p, parts, f.segments, loss, lse, st);
    }
    const void *x = p.x, *w = p.w;
    if (f.pack) {
        ProfScope s("xent_pack", st);
        if ((e = pack(p, f.depth, f.planes, ws + f.x, ws + f.w, bf16, st)) != cudaSuccess) return e;
        x = ws + f.x;
        w = ws + f.w;
    }
    Maps maps{};
    if (!encode(&maps.m[0], x, f.depth, p.N, f.planes, f.depth, 64, row_box_of(p.N)) ||
        !encode(&maps.m[1], w, f.depth, p.V, f.planes, f.depth, 64, 128))
        return cudaErrorInvalidValue;
    Args a{};
    a.p = p;
    a.row_box = row_box_of(p.N);
    a.chunks = (p.D + 63) / 64;
    a.row_tiles = tiles256(p.N);
    a.col_tiles = tiles256(p.V);
    a.unit_tiles = f.unit_tiles;
    a.units = a.row_tiles * (f.segments / 2);
    a.parts = parts;
    const int clusters = std::min(kClusters, a.units);
    {
        ProfScope s("xent_fwd", st);
        set_combos(&a, f.planes, f.planes);
        e = f.wide ? launch<kForward, 1, true, false>(a, maps, clusters, st)
            : resident(a) ? launch<kForward, 1, false, true>(a, maps, clusters, st)
                          : launch<kForward, 1, false, false>(a, maps, clusters, st);
    }
    if (e != cudaSuccess) return e;
    ProfScope s("xent_join", st);
    return launch_join_segments(p, a.parts, f.segments, loss, lse, st);
}

// Divides the products' chunks among the clusters and returns how many take
// part: dx and dw get clusters by their work, with a tile's own cost counted as
// `tile` chunks, and no part of a tile is below `least` chunks.
static int share_products(Args* a, int dx_rows, int dw_rows, int col_tiles, int dx_chunks, int dw_chunks, bool wide) {
    const int tile = wide ? 3 : 8, least = wide ? 4 : 12;
    const double cost_dx = (double)dx_rows * (dx_chunks + tile), cost_dw = (double)dw_rows * (dw_chunks + tile);
    int clusters[2];
    clusters[0] = std::max(1, std::min(kClusters - 1, (int)(kClusters * cost_dx / (cost_dx + cost_dw) + 0.5)));
    if (!a->dx) clusters[0] = 0;
    if (!a->dw) clusters[0] = kClusters;
    clusters[1] = kClusters - clusters[0];
    for (int p = 0; p < 2; ++p) {
        if (clusters[p] == 0) continue;            // not asked for
        const int rows = p ? dw_rows : dx_rows, chunks = p ? dw_chunks : dx_chunks;
        const int by_two = col_tiles % 2 == 0 ? 2 : col_tiles % 3 == 0 ? 3 : 1;
        const int siblings = clusters[p] >= by_two ? by_two : 1;
        const int tiles = rows * (col_tiles / siblings);
        int groups = clusters[p] / siblings;
        groups = (int)std::min<long long>(groups, (long long)tiles * std::max(1, chunks / least));
        a->prob[p] = Product{p ? a->cols : a->p.N, col_tiles, chunks, tiles, siblings};
        a->snap[p] = (int)std::min<long long>(wide ? 4 : 16, (long long)tiles * chunks / groups / 4);
        clusters[p] = groups * siblings;
    }
    a->first_dw = clusters[0];
    return clusters[0] + clusters[1];
}

// g of a piece is held in memory for the two products: at most 512 MiB of it, at
// least 256 columns (16384 rows, 512 wide, 32768 columns: products of 678 us in all;
// 791 us with pieces of 256 MiB, 650 us with one piece of 1 GiB).
BwdPlan plan_backward(int N, int D, int V, bool bf16) {
    BwdPlan f{};
    f.way = way_of(N, D, V, bf16);
    if (f.way == Way::kStream) {
        f.ranges = stream_blocks(V);
    } else if (f.way == Way::kFewRows) {
        f.ranges = few_rows_ranges(N, D, V, bf16);
        f.partials = up256((size_t)few_rows_tokens(N) * V * 4);     // after g
    }
    if (f.way != Way::kTiles) {
        f.total = f.partials + up256((size_t)f.ranges * N * D * 4);
        return f;
    }
    plan_operands(N, D, bf16, &f.pack, &f.planes, &f.depth);
    f.wide = several_planes(N, D, V, bf16);
    f.g_planes = f.wide ? 3 : 1;
    const long long fit = (512ll << 20) / (2ll * f.g_planes * std::max(N, 1)) / 256 * 256;
    f.cols = (int)std::min<long long>(V, std::max(256ll, fit));
    f.blocks = !f.wide && D > 256 ? 2 : 1;
    f.ldg = (f.cols + 7) / 8 * 8;
    size_t off = 0;
    const auto take = [&](size_t n) { const size_t at = off; off += up256(n); return at; };
    f.x = take(f.pack ? (size_t)f.planes * N * f.depth * 2 : 0);
    f.w = take(f.pack ? (size_t)f.planes * V * f.depth * 2 : 0);
    f.g = take((size_t)f.g_planes * N * f.ldg * 2);
    f.dx_acc = take(f.cols < V ? (size_t)N * D * 4 : 0);
    f.partials = take((size_t)kClusters * 2 * f.blocks * 256 * 256 * 4);
    f.maxima = N <= 4096 ? 0 : std::min(152, N / 2048);       // few rows: every block looks at all of them
    f.scale = take((size_t)(1 + f.maxima) * 4);
    f.total = off;
    return f;
}

cudaError_t run_backward(const Problem& p, const BwdPlan& f, char* ws, bool bf16, const float* lse, const float* dloss, void* dx,
                         void* dw, cudaStream_t st) {
    float *g = reinterpret_cast<float*>(ws + f.g), *parts = reinterpret_cast<float*>(ws + f.partials);
    if (f.way == Way::kStream) return launch_stream_gradient(p, lse, dloss, dx, dw, parts, f.ranges, bf16, st);
    if (f.way == Way::kFewRows) return launch_few_rows_gradient(p, lse, dloss, dx, dw, g, parts, f.ranges, bf16, st);
    const void *x = p.x, *w = p.w;
    cudaError_t e;
    if (f.pack) {
        ProfScope s("xent_pack", st);
        if ((e = pack(p, f.depth, f.planes, ws + f.x, ws + f.w, bf16, st)) != cudaSuccess) return e;
        x = ws + f.x;
        w = ws + f.w;
    }
    Maps logits{}, products{};
    if (!encode(&logits.m[0], x, f.depth, p.N, f.planes, f.depth, 64, row_box_of(p.N)) ||
        !encode(&logits.m[1], w, f.depth, p.V, f.planes, f.depth, 64, 128) ||
        !encode(&products.m[1], w, f.depth, p.V, f.planes, f.depth, 64, 64) ||
        !encode(&products.m[3], x, f.depth, p.N, f.planes, f.depth, 64, 64))
        return cudaErrorInvalidValue;
    Args a{};
    a.p = p;
    a.row_box = row_box_of(p.N);
    a.lse = lse;
    a.dloss = dloss;
    a.out_cols = p.D;
    // equal tiles of at most 256 * blocks columns: 712 goes as 384 and 328, not as 512 and 200
    const int d_tiles = (p.D + 256 * f.blocks - 1) / (256 * f.blocks);
    a.tile_cols = ((p.D + d_tiles - 1) / d_tiles + 31) / 32 * 32;
    a.out_f32 = !bf16;
    a.partials = parts;
    a.scale = reinterpret_cast<float*>(ws + f.scale);
    a.dx_acc = reinterpret_cast<float*>(ws + f.dx_acc);
    a.dx = dx;
    a.dw = dw;
    if (f.maxima > 0) {
        ProfScope s("xent_maxima", st);
        float* maxima = reinterpret_cast<float*>(ws + f.scale) + 1;
        a.maxima = maxima;
        a.n_maxima = f.maxima;
        e = launch_kernel(maxima_kernel, dim3(f.maxima), dim3(256), 0, st, p, dloss, maxima);
        if (e != cudaSuccess) return e;
    }
    for (int v0 = 0; v0 < p.V; v0 += f.cols) {
        const int cols = std::min(f.cols, p.V - v0);
        if (!encode(&logits.m[2], ws + f.g, cols, p.N, f.g_planes, f.ldg, 64, 32) ||
            !encode(&products.m[0], ws + f.g, cols, p.N, f.g_planes, f.ldg, 64, row_box_of(p.N)) ||
            !encode(&products.m[2], ws + f.g, cols, p.N, f.g_planes, f.ldg, 64, 64))
            return cudaErrorInvalidValue;
        a.v0 = v0;
        a.cols = cols;
        a.chunks = (p.D + 63) / 64;
        a.row_tiles = tiles256(p.N);
        a.col_tiles = tiles256(cols);
        a.unit_tiles = unit_tiles_of(a.row_tiles, a.col_tiles);
        a.units = a.row_tiles * ((a.col_tiles + a.unit_tiles - 1) / a.unit_tiles);
        {
            ProfScope s("xent_grad", st);
            const int clusters = std::min(kClusters, a.units);
            set_combos(&a, f.planes, f.planes);
            e = f.wide ? launch<kGradient, 1, true, false>(a, logits, clusters, st)
                : resident(a) ? launch<kGradient, 1, false, true>(a, logits, clusters, st)
                              : launch<kGradient, 1, false, false>(a, logits, clusters, st);
        }
        if (e != cudaSuccess) return e;
        const int workers =
            share_products(&a, tiles256(p.N), tiles256(cols), d_tiles, (cols + 63) / 64, (p.N + 63) / 64, f.wide);
        a.dx_add = v0 > 0;
        a.dx_done = v0 + cols >= p.V;
        {
            ProfScope s("xent_products", st);
            set_combos(&a, f.g_planes, f.planes);
            e = f.wide ? launch<kProducts, 1, true, false>(a, products, workers, st)
                : f.blocks == 2 ? launch<kProducts, 2, false, false>(a, products, workers, st)
                          : launch<kProducts, 1, false, false>(a, products, workers, st);
        }
        if (e != cudaSuccess) return e;
        SplitTiles splits;
        find_splits(a, workers, &splits);
        if (splits.count > 0) {
            ProfScope s("xent_join_products", st);
            const dim3 grid(splits.count, 2 * f.blocks * kEpilogueWarps);
            e = f.wide ? launch_kernel(join_products_kernel<1, true>, grid, dim3(512), 0, st, a, splits)
                : f.blocks == 2 ? launch_kernel(join_products_kernel<2, false>, grid, dim3(512), 0, st, a, splits)
                                : launch_kernel(join_products_kernel<1, false>, grid, dim3(512), 0, st, a, splits);
            if (e != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

}  // namespace xent
}  // namespace fibattn
