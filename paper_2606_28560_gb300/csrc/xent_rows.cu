// xent_rows.cu -- the cross entropy for three to 32 rows (a small batch over a large
// head), and the joins of per-row statistics and of dx's parts.
//
// With few rows the work is w read once per pass, and fp32 cannot afford to be
// split into planes in memory for the fifth-generation cores.  These kernels are
// streams over w: every warp takes sixteen rows of w at a time straight from memory into
// the operand registers of mma.sync (tf32, 16 x 8 x 8), against up to 32 rows of x
// in shared memory.  fp32 values go as two tf32 values, x = hi + lo, three products
// of the four (the fourth is below 2^-22); bf16 values are exact.  The large
// products are summed 64 deep before they are added in fp32, because the tensor
// core truncates.
//
// Bound by memory in bf16 and up to 16 rows in fp32: 16 x 2048 x 131072 in fp32 takes
// 193 us forward (5.6 TB/s) and 633 backward (2 x 1.07 GB read, 1.07 written).
// With 32 rows, 361 and 1040, it is halfway between memory (159 and 476) and the
// tensor rate (150 T multiplications a second, three for one in fp32): what is
// issued beside them, the splitting in two and the loads of x, is the rest.
//
// A sum does not care for the order of its terms, so lanes take them as memory
// gives them: in the logits a lane's depth values are consecutive; in the
// products a lane's four columns are, and its tokens.
#include <algorithm>

#include "xent.cuh"

namespace fibattn {
namespace xent {
namespace {

constexpr int kWarps = 8;
constexpr int kTileRows = 16;                      // rows of w in a warp's hands

template <typename T> struct Lane { static constexpr int kValues = 16 / sizeof(T); };   // of 16 bytes

// The 16 bytes at p, n values of them (zeros past them).  VECTORS: 16-byte
// boundaries, and n is 0 or less or all or more.
template <typename T, bool VECTORS> __device__ __forceinline__ uint4 fetch16(const T* p, int n) {
    if constexpr (VECTORS) {
        return n > 0 ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
    } else {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = i < n ? __float_as_uint(p[i]) : 0u;
            } else {
                const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
                w[i] = (2 * i < n ? (unsigned)q[2 * i] : 0u) | (2 * i + 1 < n ? (unsigned)q[2 * i + 1] << 16 : 0u);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T> __device__ __forceinline__ void unfold(const uint4& u, float* x) {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
// Four values at p, of which n are there.  VECTORS: all or none, aligned to them.
template <typename T, bool VECTORS> __device__ __forceinline__ void load4(const T* p, int n, float* x) {
    if (VECTORS && n > 0) {
        if constexpr (sizeof(T) == 4) {
            const float4 v = *reinterpret_cast<const float4*>(p);
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
            x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = !VECTORS && j < n ? to_f(p[j]) : 0.f;
}
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }
template <typename T, bool VECTORS> __device__ __forceinline__ void store4(T* p, int n, const float* x) {
    if constexpr (!VECTORS) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) put(p + j, x[j]);
    } else if (n > 0) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
            const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
            *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
        }
    }
}

// N consecutive fp32 values, aligned to all of them (to 16 bytes at most), or zeros.
template <int N> __device__ __forceinline__ void load_together(const float* p, bool there, float* x) {
#pragma unroll
    for (int i = 0; i < N; i += N < 4 ? N : 4) {
        if constexpr (N == 1) {
            x[i] = there ? *p : 0.f;
        } else if constexpr (N == 2) {
            const float2 v = there ? *reinterpret_cast<const float2*>(p) : make_float2(0.f, 0.f);
            x[i] = v.x; x[i + 1] = v.y;
        } else {
            const float4 v = there ? *reinterpret_cast<const float4*>(p + i) : make_float4(0.f, 0.f, 0.f, 0.f);
            x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
        }
    }
}

// The tf32 value (11 bits) next to x, ties away from zero, with integer operations:
// conversion instructions go at an eighth of their rate, as many of them would take
// as long as the products.  Of a NaN whose payload overflows here, low() is a NaN.
__device__ __forceinline__ unsigned high(float x) { return (__float_as_uint(x) + 0x1000u) & 0xffffe000u; }
// The same for values of w, of which a mask may be the lowest fp32 value or an infinity:
// tf32's largest value with their sign, what is left (an infinity's: itself) to low().
// (Forward and backward of 16 x 2048 x 131072 in fp32 822 us instead of 813, of 32 rows
// 1400 instead of 1340.)
__device__ __forceinline__ unsigned high_of_weight(float x) {
    float r;
    asm("min.NaN.xorsign.abs.f32 %0, %1, %2;\n" : "=f"(r) : "f"(x), "f"(__uint_as_float(0x7f7fe000u)));
    return high(r);
}
__device__ __forceinline__ unsigned low(float x, unsigned hi) { return __float_as_uint(x - __uint_as_float(hi)); }

__device__ __forceinline__ void mma(float* c, const unsigned* a, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Of x's blocks of depth (four lanes' 16 bytes), those that a block of threads can
// hold for oct x 8 rows.
constexpr size_t kMostSmem = 224 * 1024;           // of the 227 KB that it may have, two for statistics
template <typename T> __host__ __device__ constexpr int staged_blocks(int oct, int D) {
    const int block = 4 * Lane<T>::kValues, all = (D + block - 1) / block, most = (int)(kMostSmem / ((size_t)oct * 8 * block * 4));
    return all < most ? all : most;
}

// Where value j of lane l's 16 bytes of block b of octet o's rows of x lies.
template <typename T, int OCT> __device__ __forceinline__ int staged(int b, int o, int l, int j) {
    return (((b * OCT + o) * (Lane<T>::kValues / 4) + j / 4) * 32 + l) * 4 + j % 4;
}

// Logits of 16 rows of w (from v0) and OCT x 8 rows of x (xs):
// s[o][0..3] = rows g, g, g + 8, g + 8 and tokens 2 t, 2 t + 1, 2 t, 2 t + 1 of
// octet o, lane = 4 g + t.  x: the same rows in memory, `rows` of them, read where they
// are deeper than what is staged (never when WHOLE).  AHEAD: w is asked into L2 two
// steps before it is loaded.
template <typename T, int OCT, bool VECTORS, bool WHOLE, bool AHEAD>
__device__ __forceinline__ void tile_logits(const T* w, int V, int D, int v0, const float* xs, const T* x, int rows, int lane,
                                            float (*s)[4]) {
    constexpr int kVal = Lane<T>::kValues, kBlock = 4 * kVal, kAhead = 4;   // blocks of depth under way
    constexpr bool kExact = sizeof(T) == 2;
    const int g = lane >> 2, t = lane & 3, blocks = (D + kBlock - 1) / kBlock;
    const T* r0 = w + (size_t)(v0 + g) * D + t * kVal;
    const T* r1 = r0 + (size_t)8 * D;
    const bool in0 = v0 + g < V, in1 = v0 + g + 8 < V;
    float small[OCT][4];
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[o][j] = small[o][j] = 0.f;
    uint4 n0[kAhead], n1[kAhead];                  // the next blocks, as they come
    const auto fetch = [&](int b0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = (b0 + u) * kBlock, left = D - k - t * kVal;
            n0[u] = fetch16<T, VECTORS>(r0 + k, in0 ? left : 0);
            n1[u] = fetch16<T, VECTORS>(r1 + k, in1 ? left : 0);
        }
        if constexpr (AHEAD) {                     // 256 bytes of each row, of the next tile's too
            constexpr int kStep = kAhead * kBlock;
            const int depth = (blocks + kAhead - 1) / kAhead * kStep;
            int k = b0 * kBlock + 2 * kStep + (lane >> 4) * (kStep / 2), v = v0 + (lane & 15);
            if (k >= depth) { k -= depth; v += kTileRows; }
            if (k < D && v < V) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(w + (size_t)v * D + k));
        }
    };
    fetch(0);
    for (int b0 = 0; b0 < blocks; b0 += kAhead) {
        float a0[kAhead][kVal], a1[kAhead][kVal];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            unfold<T>(n0[u], a0[u]);
            unfold<T>(n1[u], a1[u]);
        }
        if (b0 + kAhead < blocks) fetch(b0 + kAhead);
        float big[OCT][4];                         // 64 (fp32) or 128 (bf16) deep
#pragma unroll
        for (int o = 0; o < OCT; ++o)
#pragma unroll
            for (int j = 0; j < 4; ++j) big[o][j] = 0.f;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (b0 + u < blocks) {
#pragma unroll
                for (int q = 0; q < kVal / 4; ++q) {
                    unsigned ah[2][4], al[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // two steps of eight: values 4 q + 2 h, 4 q + 2 h + 1
                        const float e[4] = {a0[u][4 * q + 2 * h], a1[u][4 * q + 2 * h], a0[u][4 * q + 2 * h + 1],
                                            a1[u][4 * q + 2 * h + 1]};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            ah[h][j] = kExact ? __float_as_uint(e[j]) : high_of_weight(e[j]);
                            al[h][j] = kExact ? 0u : low(e[j], ah[h][j]);
                        }
                    }
#pragma unroll
                    for (int o = 0; o < OCT; ++o) {
                        float e[4];
                        if (WHOLE || b0 + u < staged_blocks<T>(OCT, D)) {
                            const float4 f = *reinterpret_cast<const float4*>(xs + staged<T, OCT>(b0 + u, o, lane, 4 * q));
                            e[0] = f.x; e[1] = f.y; e[2] = f.z; e[3] = f.w;
                        } else {
                            const int n = 8 * o + g, k = (b0 + u) * kBlock + t * kVal + 4 * q;
                            load4<T, VECTORS>(x + (size_t)n * D + k, n < rows ? D - k : 0, e);
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const unsigned b0h = kExact ? __float_as_uint(e[2 * h]) : high(e[2 * h]);
                            const unsigned b1h = kExact ? __float_as_uint(e[2 * h + 1]) : high(e[2 * h + 1]);
                            if (!kExact) {
                                mma(small[o], al[h], b0h, b1h);
                                mma(small[o], ah[h], low(e[2 * h], b0h), low(e[2 * h + 1], b1h));
                            }
                            mma(big[o], ah[h], b0h, b1h);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int o = 0; o < OCT; ++o)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[o][j] += big[o][j];
    }
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[o][j] += small[o][j];
}

// x's rows from n0 (8 OCT of them, zeros past N), as deep as they fit, into shared memory,
// as tile_logits reads them, 16 bytes to a thread, eight of them under way.
template <typename T, int OCT, bool VECTORS, int WARPS>
__device__ __forceinline__ void stage_x(const Problem& p, int n0, float* xs) {
    constexpr int kVal = Lane<T>::kValues, kBlock = 4 * kVal, kAhead = 8;
    const int pieces = staged_blocks<T>(OCT, p.D) * OCT * 32;
    for (int i0 = threadIdx.x; i0 < pieces; i0 += kAhead * 32 * WARPS) {
        uint4 u[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * 32 * WARPS, l = i & 31, n = n0 + i / 32 % OCT * 8 + l / 4, c = i / (32 * OCT) * kBlock + l % 4 * kVal;
            u[k] = fetch16<T, VECTORS>(static_cast<const T*>(p.x) + (size_t)n * p.D + c, n < p.N ? p.D - c : 0);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * 32 * WARPS;
            float e[kVal];
            unfold<T>(u[k], e);
#pragma unroll
            for (int j = 0; j < kVal; j += 4)
                if (i < pieces)
                    *reinterpret_cast<float4*>(xs + staged<T, OCT>(i / (32 * OCT), i / 32 % OCT, i & 31, j)) =
                        make_float4(e[j], e[j + 1], e[j + 2], e[j + 3]);
        }
    }
}

__device__ __forceinline__ void merge(float& m, float& l, float m2, float l2) {
    const float top = fmaxf(m, m2), ms = top == -INFINITY ? 0.f : top;
    l = l * expf(m - ms) + l2 * expf(m2 - ms);
    m = top;
}

// Whether tile_logits asks ahead: for eight deep rows it is memory's latency that bounds,
// otherwise the instructions are missed elsewhere (fp32, us forward and backward, with
// / without: 8 x 8192 x 20000 609 / 653, 8 x 7168 x 20000 475 / 492, 16 x 2048 x
// 131072 833 / 823, 16 x 512 x 32768 74 / 73).
constexpr bool asked_ahead(int oct, int warps) { return oct == 1 && warps == 16; }

// Block: a segment of w (for `groups` > 1 as many groups of 8 OCT rows of x, whose
// blocks follow one another so that they read w together).  Statistics
// [row][segment].
template <typename T, int OCT, bool VECTORS, int WARPS, bool WHOLE>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS) rows_kernel(Problem p, FwdParts parts, int segments, int groups) {
    extern __shared__ __align__(16) float xs[];
    __shared__ float red[2][WARPS][8 * OCT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int seg = blockIdx.x / groups, n0 = blockIdx.x % groups * 8 * OCT;
    grid_dependency_sync();
    stage_x<T, OCT, VECTORS, WARPS>(p, n0, xs);
    float m[OCT][2], l[OCT][2];
    int target[OCT][2];
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = n0 + 8 * o + 2 * t + j;
            target[o][j] = n < p.N ? target_column(p, n) : kIgnored;
            m[o][j] = -INFINITY;
            l[o][j] = 0.f;
        }
    __syncthreads();
    const int tiles = (p.V + kTileRows - 1) / kTileRows, worker = seg * WARPS + warp, workers = segments * WARPS;
    for (int i = (int)((long long)tiles * worker / workers); i < (int)((long long)tiles * (worker + 1) / workers); ++i) {
        float s[OCT][4];
        tile_logits<T, OCT, VECTORS, WHOLE, asked_ahead(OCT, WARPS)>(static_cast<const T*>(p.w), p.V, p.D, i * kTileRows, xs,
                                                                               static_cast<const T*>(p.x) + (size_t)n0 * p.D,
                                                                               p.N - n0, lane, s);
        const int v = i * kTileRows + g;
#pragma unroll
        for (int o = 0; o < OCT; ++o)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (v == target[o][j]) parts.target_logit[n0 + 8 * o + 2 * t + j] = s[o][j];
                if (v + 8 == target[o][j]) parts.target_logit[n0 + 8 * o + 2 * t + j] = s[o][2 + j];
                const float a = v < p.V ? s[o][j] : -INFINITY, b = v + 8 < p.V ? s[o][2 + j] : -INFINITY;
                const float top = fmaxf(m[o][j], fmaxf(a, b)), ms = top == -INFINITY ? 0.f : top;
                l[o][j] = l[o][j] * expf(m[o][j] - ms) + (expf(a - ms) + expf(b - ms));
                m[o][j] = top;
            }
    }
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2)
                merge(m[o][j], l[o][j], __shfl_xor_sync(0xffffffffu, m[o][j], d), __shfl_xor_sync(0xffffffffu, l[o][j], d));
            if (g == 0) {
                red[0][warp][8 * o + 2 * t + j] = m[o][j];
                red[1][warp][8 * o + 2 * t + j] = l[o][j];
            }
        }
    __syncthreads();
    if ((int)threadIdx.x < 8 * OCT && n0 + (int)threadIdx.x < p.N) {
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) merge(top, sum, red[0][i][threadIdx.x], red[1][i][threadIdx.x]);
        parts.m[(size_t)(n0 + threadIdx.x) * segments + seg] = top;
        parts.l[(size_t)(n0 + threadIdx.x) * segments + seg] = sum;
    }
}

// The same logits, as g[v][token] (row length `tokens`; zeros for tokens past N).
template <typename T, int OCT, bool VECTORS, int WARPS, bool WHOLE>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS)
rows_gradient_kernel(Problem p, const float* lse, const float* dloss, float* gradient, int tokens, int groups) {
    extern __shared__ __align__(16) float xs[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int seg = blockIdx.x / groups, n0 = blockIdx.x % groups * 8 * OCT;
    grid_dependency_sync();
    stage_x<T, OCT, VECTORS, WARPS>(p, n0, xs);
    int target[OCT][2];
    float z[OCT][2], dl[OCT][2];
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = n0 + 8 * o + 2 * t + j;
            target[o][j] = n < p.N ? target_column(p, n) : kIgnored;
            z[o][j] = target[o][j] >= 0 ? lse[n] : 0.f;
            dl[o][j] = target[o][j] >= 0 ? dloss[n] : 0.f;
            if (target[o][j] == kBad && seg == 0 && warp == 0 && g == 0) raise_status(p.status, kStatusTarget);
        }
    __syncthreads();
    const int tiles = (p.V + kTileRows - 1) / kTileRows, worker = seg * WARPS + warp, workers = gridDim.x / groups * WARPS;
    for (int i = (int)((long long)tiles * worker / workers); i < (int)((long long)tiles * (worker + 1) / workers); ++i) {
        float s[OCT][4];
        tile_logits<T, OCT, VECTORS, WHOLE, asked_ahead(OCT, WARPS)>(static_cast<const T*>(p.w), p.V, p.D, i * kTileRows, xs,
                                                                               static_cast<const T*>(p.x) + (size_t)n0 * p.D,
                                                                               p.N - n0, lane, s);
#pragma unroll
        for (int o = 0; o < OCT; ++o)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int v = i * kTileRows + g + 8 * h;
                float2 out;
                float* e = &out.x;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    e[j] = target[o][j] < 0 ? 0.f : dl[o][j] * (expf(s[o][2 * h + j] - z[o][j]) - (v == target[o][j] ? 1.f : 0.f));
                if (v < p.V) *reinterpret_cast<float2*>(gradient + (size_t)v * tokens + n0 + 8 * o + 2 * t) = out;
            }
    }
}

// dw[v] = sum_n g[v][n] x[n] and dx[n] = sum_v g[v][n] w[v].  A warp takes 32
// columns of a range of rows of w, sixteen rows at a time.  Lane 4 g + t has the
// consecutive columns 4 g .. 4 g + 3: rows g and g + 8 of two operands of 16 rows.
//   dx^T (columns x tokens) += w^T (columns x 8 rows of w) g (8 rows x tokens)
//   dw^T (columns x 8 rows of w) = x^T (columns x tokens) g^T (tokens x 8 rows)
// In the first, token OCT g + o is column g of octet o; in the second,
// tokens 2 OCT t + 2 o and + 1 are depth t and t + 4 of octet o.
// parts[range][n][D]: dx over the range.
//
// Registers allow one to three blocks to an SM, too few loads under way for memory's
// latency: the rows of w four tiles ahead are asked into L2, the next tile's g into
// L1 (fp32, 32 x 2048 x 131072: 904 us without, 763 with the first, 705 with both).
template <typename T> constexpr int resident(int oct) { return oct == 4 ? 1 : oct == 1 && sizeof(T) == 2 ? 3 : 2; }

template <typename T, int OCT, bool VECTORS>
__global__ void __launch_bounds__(32 * kWarps, resident<T>(OCT))
rows_products_kernel(Problem p, const float* gradient, T* dw, float* parts, int ranges) {
    constexpr bool kExact = sizeof(T) == 2;
    constexpr int kTokens = 8 * OCT;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int unit = blockIdx.x * kWarps + (threadIdx.x >> 5), column_groups = (p.D + 31) / 32;
    grid_dependency_sync();
    if (unit >= column_groups * ranges) return;
    // neighbouring warps: the column groups of the same rows
    const int c = unit % column_groups * 32 + 4 * g, range = unit / column_groups;
    const int left = p.D - c;
    float x[OCT][2][4];
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = 2 * OCT * t + 2 * o + h;
            load4<T, VECTORS>(static_cast<const T*>(p.x) + (size_t)n * p.D + c, n < p.N ? left : 0, x[o][h]);
        }
    float dx[2][OCT][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int o = 0; o < OCT; ++o)
#pragma unroll
            for (int j = 0; j < 4; ++j) dx[i][o][j] = 0.f;
    const T* w = static_cast<const T*>(p.w);
    const int tiles = (p.V + kTileRows - 1) / kTileRows;
    const int lo = (int)((long long)tiles * range / ranges), hi = (int)((long long)tiles * (range + 1) / ranges);
    constexpr int kL2Ahead = 4;
    float next[4][4];                              // the next tile's rows of w
    const auto fetch = [&](int v0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {              // rows v0 + 4 u + t
            const int v = v0 + 4 * u + t;
            load4<T, VECTORS>(w + (size_t)v * p.D + c, v < p.V ? left : 0, next[u]);
        }
        const int v = v0 + kL2Ahead * kTileRows + (lane & 15);
        if (lane < 16 && v < p.V) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(w + (size_t)v * p.D + (c - 4 * g)));
        const int vg = v0 + kTileRows + (lane & 15);
        if (lane < 16 && vg < p.V) asm volatile("prefetch.global.L1 [%0];\n" ::"l"(gradient + (size_t)vg * kTokens));
    };
    if (lo < hi) fetch(lo * kTileRows);
    for (int i0 = lo; i0 < hi; ++i0) {
        const int v0 = i0 * kTileRows;
        float a[4][4], gv[4][OCT], gt[2][2 * OCT];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) a[u][j] = next[u][j];
        if (i0 + 1 < hi) fetch(v0 + kTileRows);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int v = v0 + 4 * u + t;
            const float* q = gradient + (size_t)v * kTokens + OCT * g;
            load_together<OCT>(q, v < p.V, gv[u]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {              // row v0 + 8 h + g, this lane's tokens
            const int v = v0 + 8 * h + g;
            const float* q = gradient + (size_t)v * kTokens + 2 * OCT * t;
            load_together<2 * OCT>(q, v < p.V, gt[h]);
        }
        if (parts) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float sum[OCT][4];
#pragma unroll
                for (int o = 0; o < OCT; ++o)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[o][j] = 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {      // eight rows of w: 4 u + t with u = 2 h, 2 h + 1
                    const float e[4] = {a[2 * h][2 * i], a[2 * h][2 * i + 1], a[2 * h + 1][2 * i], a[2 * h + 1][2 * i + 1]};
                    unsigned ah[4], al[4], bh[OCT][2];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        ah[j] = kExact ? __float_as_uint(e[j]) : high_of_weight(e[j]);
                        al[j] = kExact ? 0u : low(e[j], ah[j]);
                    }
#pragma unroll
                    for (int o = 0; o < OCT; ++o) {
                        bh[o][0] = high(gv[2 * h][o]);
                        bh[o][1] = high(gv[2 * h + 1][o]);
                        mma(sum[o], ah, low(gv[2 * h][o], bh[o][0]), low(gv[2 * h + 1][o], bh[o][1]));
                    }
                    if (!kExact) {
#pragma unroll
                        for (int o = 0; o < OCT; ++o) mma(sum[o], al, bh[o][0], bh[o][1]);
                    }
#pragma unroll
                    for (int o = 0; o < OCT; ++o) mma(sum[o], ah, bh[o][0], bh[o][1]);
                }
#pragma unroll
                for (int o = 0; o < OCT; ++o)
#pragma unroll
                    for (int j = 0; j < 4; ++j) dx[i][o][j] += sum[o][j];
            }
        }
        if (dw) {
            float out[2][2][4];                    // [rows v0 + 8 h ..][columns 2 i ..]
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) out[h][i][j] = 0.f;
#pragma unroll
            for (int o = 0; o < OCT; ++o) {
                unsigned ah[2][4], al[2][4], bh[2][2], bl[2][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = x[o][j / 2][2 * i + j % 2];
                        ah[i][j] = kExact ? __float_as_uint(e) : high(e);
                        al[i][j] = kExact ? 0u : low(e, ah[i][j]);
                    }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        bh[h][j] = high(gt[h][2 * o + j]);
                        bl[h][j] = low(gt[h][2 * o + j], bh[h][j]);
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k) mma(out[k / 2][k % 2], ah[k % 2], bl[k / 2][0], bl[k / 2][1]);
                if (!kExact) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma(out[k / 2][k % 2], al[k % 2], bh[k / 2][0], bh[k / 2][1]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) mma(out[k / 2][k % 2], ah[k % 2], bh[k / 2][0], bh[k / 2][1]);
            }
            // columns 4 g .. 4 g + 3 of rows 2 t and 2 t + 1
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int v = v0 + 8 * h + 2 * t + j;
                    const float r[4] = {out[h][0][j], out[h][0][2 + j], out[h][1][j], out[h][1][2 + j]};
                    if (v < p.V) store4<T, VECTORS>(dw + (size_t)v * p.D + c, left, r);
                }
        }
    }
    if (!parts) return;
    // dx^T: columns 4 g + 2 i, 4 g + 2 i + 1; tokens OCT (2 t + j) + o
#pragma unroll
    for (int o = 0; o < OCT; ++o)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = OCT * (2 * t + j) + o;
            const float r[4] = {dx[0][o][j], dx[0][o][2 + j], dx[1][o][j], dx[1][o][2 + j]};
            if (n < p.N) store4<float, VECTORS>(parts + ((size_t)range * p.N + n) * p.D + c, left, r);
        }
}

__device__ __forceinline__ void finish_row(const Problem& p, const FwdParts& parts, int n, float z, float* loss, float* lse) {
    lse[n] = z;
    const int t = target_column(p, n);
    if (t == kBad) raise_status(p.status, kStatusTarget);
    loss[n] = t == kIgnored ? 0.f : t == kBad ? NAN : z - parts.target_logit[n];
}

// dx[n][c] = sum over the ranges of parts[range][n][c]: 32 columns to a block of
// 256 threads, every eighth part to a thread.
template <typename T> __global__ void __launch_bounds__(256) join_dx_kernel(const float* parts, int ranges, long long values, T* dx) {
    __shared__ float red[8][32];
    grid_dependency_sync();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const long long i = blockIdx.x * 32ll + lane;
    float s = 0.f;
    if (i < values) {
#pragma unroll 8
        for (int b = part; b < ranges; b += 8) s += parts[b * values + i];
    }
    red[part][lane] = s;
    __syncthreads();
    if (part == 0 && i < values) {
        s = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) s += red[k][lane];
        put(dx + i, s);
    }
}

// Many rows: eight threads each, every eighth segment of [segment][row]; a
// block takes 32 rows, so that a warp reads 128 consecutive bytes.
__global__ void __launch_bounds__(256) join_segments_kernel(Problem p, FwdParts parts, int segments, float* loss, float* lse) {
    __shared__ float red[2][8][32];
    grid_dependency_sync();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, n = blockIdx.x * 32 + lane;
    float m = -INFINITY, l = 0.f;
    if (n < p.N) {
#pragma unroll 4
        for (int s = part; s < segments; s += 8) {
            const float a = parts.m[(size_t)s * p.N + n], b = parts.l[(size_t)s * p.N + n];
            const float top = fmaxf(m, a), ms = top == -INFINITY ? 0.f : top;
            l = l * expf(m - ms) + b * expf(a - ms);
            m = top;
        }
    }
    red[0][part][lane] = m;
    red[1][part][lane] = l;
    __syncthreads();
    if (part == 0 && n < p.N) {
        float top = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, red[0][i][lane]);
        const float ms = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int i = 0; i < 8; ++i) l += red[1][i][lane] * expf(red[0][i][lane] - ms);
        finish_row(p, parts, n, top + logf(l), loss, lse);
    }
}

// Few rows: a block of 256 threads each, statistics [row][segment].
__global__ void __launch_bounds__(256) join_rows_kernel(Problem p, FwdParts parts, int segments, float* loss, float* lse) {
    __shared__ float red[2][8];
    grid_dependency_sync();
    const int n = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float* pm = parts.m + (size_t)n * segments;
    const float* pl = parts.l + (size_t)n * segments;
    float m = -INFINITY, l = 0.f;
    for (int s = threadIdx.x; s < segments; s += 256) {
        const float a = pm[s], b = pl[s], top = fmaxf(m, a), ms = top == -INFINITY ? 0.f : top;
        l = l * expf(m - ms) + b * expf(a - ms);
        m = top;
    }
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float ms = top == -INFINITY ? 0.f : top;
    l *= expf(m - ms);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) {
        red[0][warp] = top;
        red[1][warp] = l;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        top = -INFINITY;
        l = 0.f;
        for (int i = 0; i < 8; ++i) top = fmaxf(top, red[0][i]);
        ms = top == -INFINITY ? 0.f : top;
        for (int i = 0; i < 8; ++i) l += red[1][i] * expf(red[0][i] - ms);
        finish_row(p, parts, n, top + logf(l), loss, lse);
    }
}

template <typename K> cudaError_t allow_smem(K kern) {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
}

// x of oct x 8 rows, whole (its values are fp32 there, its depth a multiple of 32).
size_t smem_of(int oct, int D) { return (size_t)oct * 8 * ((D + 31) / 32 * 32) * 4; }

// Octets of rows of x: 1, 2 or 4, as many as there are; and how many a block takes at a
// time: two if they fit its shared memory (of one, the rest is read where it lies:
// D > 7168).
int octets(int N) { return N <= 8 ? 1 : N <= 16 ? 2 : 4; }
int octets_at_once(int N, int D) { return N > 8 && smem_of(2, D) <= kMostSmem ? 2 : 1; }

// Blocks of eight warps while two of them fit an SM, else one of sixteen.
bool sixteen_warps(int oct, int D) { return smem_of(oct, D) > 100 * 1024; }

template <typename T, int OCT, bool VECTORS, int WARPS, bool WHOLE = true>
cudaError_t launch_rows(const Problem& p, const FwdParts& parts, int segments, cudaStream_t st) {
    const auto kern = rows_kernel<T, OCT, VECTORS, WARPS, WHOLE>;
    const cudaError_t e = allow_smem(kern);
    if (e != cudaSuccess) return e;
    const int groups = octets(p.N) / OCT;
    const size_t smem = std::min(smem_of(OCT, p.D), kMostSmem);
    return launch_kernel(kern, dim3((unsigned)(segments * groups)), dim3(32 * WARPS), smem, st, p, parts, segments, groups);
}
template <typename T, bool VECTORS>
cudaError_t rows(const Problem& p, const FwdParts& parts, int segments, cudaStream_t st) {
    switch (octets_at_once(p.N, p.D)) {
    case 1:
        return smem_of(1, p.D) > kMostSmem ? launch_rows<T, 1, VECTORS, 16, false>(p, parts, segments, st)
               : sixteen_warps(1, p.D)     ? launch_rows<T, 1, VECTORS, 16>(p, parts, segments, st)
                                           : launch_rows<T, 1, VECTORS, kWarps>(p, parts, segments, st);
    default:
        return sixteen_warps(2, p.D) ? launch_rows<T, 2, VECTORS, 16>(p, parts, segments, st)
                                     : launch_rows<T, 2, VECTORS, kWarps>(p, parts, segments, st);
    }
}

template <typename T, int OCT, bool VECTORS, int WARPS, bool WHOLE = true>
cudaError_t launch_gradient(const Problem& p, const float* lse, const float* dloss, float* gradient, cudaStream_t st) {
    const auto kern = rows_gradient_kernel<T, OCT, VECTORS, WARPS, WHOLE>;
    const cudaError_t e = allow_smem(kern);
    if (e != cudaSuccess) return e;
    const int groups = octets(p.N) / OCT;
    const size_t smem = std::min(smem_of(OCT, p.D), kMostSmem);
    ProfScope s("xent_few_rows_grad", st);
    return launch_kernel(kern, dim3((unsigned)(few_rows_segments(p.N, p.D, p.V) * groups)), dim3(32 * WARPS), smem, st, p,
                         lse, dloss, gradient, 8 * octets(p.N), groups);
}
template <typename T, int OCT, bool VECTORS>
cudaError_t launch_products(const Problem& p, const float* gradient, T* dw, float* parts, int ranges, cudaStream_t st) {
    const int units = (p.D + 31) / 32 * ranges;
    ProfScope s("xent_few_rows_products", st);
    return launch_kernel(rows_products_kernel<T, OCT, VECTORS>, dim3((unsigned)((units + kWarps - 1) / kWarps)), dim3(32 * kWarps), 0,
                         st, p, gradient, dw, parts, ranges);
}
template <typename T, bool VECTORS>
cudaError_t gradient_of(const Problem& p, const float* lse, const float* dloss, T* dx, T* dw, float* gradient, float* parts, int ranges,
                        cudaStream_t st) {
    const int once = octets_at_once(p.N, p.D);
    const bool sixteen = sixteen_warps(once, p.D);
    cudaError_t e = smem_of(1, p.D) > kMostSmem ? launch_gradient<T, 1, VECTORS, 16, false>(p, lse, dloss, gradient, st)
                    : once == 1 && sixteen      ? launch_gradient<T, 1, VECTORS, 16>(p, lse, dloss, gradient, st)
                    : once == 1                 ? launch_gradient<T, 1, VECTORS, kWarps>(p, lse, dloss, gradient, st)
                    : sixteen                   ? launch_gradient<T, 2, VECTORS, 16>(p, lse, dloss, gradient, st)
                                                : launch_gradient<T, 2, VECTORS, kWarps>(p, lse, dloss, gradient, st);
    if (e != cudaSuccess) return e;
    float* to = dx ? parts : nullptr;
    const int oct = octets(p.N);
    e = oct == 1   ? launch_products<T, 1, VECTORS>(p, gradient, dw, to, ranges, st)
        : oct == 2 ? launch_products<T, 2, VECTORS>(p, gradient, dw, to, ranges, st)
                   : launch_products<T, 4, VECTORS>(p, gradient, dw, to, ranges, st);
    return e != cudaSuccess || !dx ? e : launch_join_dx(p, parts, ranges, dx, sizeof(T) == 2, st);
}

}  // namespace

bool few_rows_applies(int N) { return N <= 32; }

int few_rows_tokens(int N) { return 8 * octets(N); }

// Segments of w: as many as fill the SMs once over the groups of rows of x (more
// would only stage x more often), and no more than leave a block tiles 1024 deep in
// all (a small w is spread over the SMs before it is over warps), eight at most.
int few_rows_segments(int N, int D, int V) {
    const int once = octets_at_once(N, D), groups = octets(N) / once, blocks = sixteen_warps(once, D) ? 152 : 2 * 152;
    const int rows = kTileRows * std::max(1, std::min(8, 1024 / D));
    return std::max(1, std::min(blocks / groups, (V + rows - 1) / rows));
}

// Ranges of rows of w in the products: as many blocks of warps as an SM holds over
// all groups of 32 columns, a tile to a warp at least.
int few_rows_ranges(int N, int D, int V, bool bf16) {
    const int groups = (D + 31) / 32, oct = octets(N), blocks = bf16 ? resident<__nv_bfloat16>(oct) : resident<float>(oct);
    return std::max(1, std::min(152 * blocks * kWarps / groups, (V + kTileRows - 1) / kTileRows));
}

cudaError_t launch_few_rows(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st) {
    if (bf16) return p.D % 8 == 0 ? rows<__nv_bfloat16, true>(p, parts, segments, st) : rows<__nv_bfloat16, false>(p, parts, segments, st);
    return p.D % 4 == 0 ? rows<float, true>(p, parts, segments, st) : rows<float, false>(p, parts, segments, st);
}

cudaError_t launch_few_rows_gradient(const Problem& p, const float* lse, const float* dloss, void* dx, void* dw, float* gradient,
                                     float* parts, int ranges, bool bf16, cudaStream_t st) {
    if (bf16) {
        auto *x = static_cast<__nv_bfloat16*>(dx), *w = static_cast<__nv_bfloat16*>(dw);
        return p.D % 8 == 0 ? gradient_of<__nv_bfloat16, true>(p, lse, dloss, x, w, gradient, parts, ranges, st)
                            : gradient_of<__nv_bfloat16, false>(p, lse, dloss, x, w, gradient, parts, ranges, st);
    }
    auto *x = static_cast<float*>(dx), *w = static_cast<float*>(dw);
    return p.D % 4 == 0 ? gradient_of<float, true>(p, lse, dloss, x, w, gradient, parts, ranges, st)
                        : gradient_of<float, false>(p, lse, dloss, x, w, gradient, parts, ranges, st);
}

cudaError_t launch_join_dx(const Problem& p, const float* parts, int ranges, void* dx, bool bf16, cudaStream_t st) {
    ProfScope s("xent_join_dx", st);
    const long long values = (long long)p.N * p.D;
    const dim3 grid((unsigned)((values + 31) / 32));
    return bf16 ? launch_kernel(join_dx_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, parts, ranges, values,
                                static_cast<__nv_bfloat16*>(dx))
                : launch_kernel(join_dx_kernel<float>, grid, dim3(256), 0, st, parts, ranges, values, static_cast<float*>(dx));
}

cudaError_t launch_join_segments(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st) {
    return launch_kernel(join_segments_kernel, dim3((p.N + 31) / 32), dim3(256), 0, st, p, parts, segments, loss, lse);
}

cudaError_t launch_join_rows(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st) {
    return launch_kernel(join_rows_kernel, dim3(p.N), dim3(256), 0, st, p, parts, segments, loss, lse);
}

}  // namespace xent
}  // namespace fibattn
