// xent_simple.cu -- linear cross entropy on the fp32 pipes: tiles of the
// products C[i][j] = sum_k A[i][k] B[j][k] of 128 x 128, eight by eight per
// thread, with the operand converted to fp32 as it is staged.  Right for every
// type, size and stride; bound by the fp32 FMA rate (two shared-memory reads
// of 32 bytes per 64 FMAs keep the pipe fed).
#include "xent.cuh"

#include <algorithm>

namespace fibattn {
namespace xent {
namespace {

constexpr int kT = 128;        // tile edge
constexpr int kK = 16;         // staged depth
constexpr int kPad = 4;

// An operand: element (i, k) at p[i * si + k * sk], zero outside rows x depth.
template <typename T> struct Operand {
    const T* p;
    long long si, sk;
    int rows, depth;
};

template <typename TA, typename TB> struct Tile {
    float c[8][8];

    // kfast: consecutive k are consecutive in memory (else consecutive i are).
    template <typename T>
    static __device__ __forceinline__ void fetch(float* r, const Operand<T>& o, int i0, int k0, bool kfast) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int e = threadIdx.x + 256 * u;
            const int i = i0 + (kfast ? e / kK : e % kT), k = k0 + (kfast ? e % kK : e / kT);
            r[u] = (i < o.rows && k < o.depth) ? to_f(o.p[i * o.si + k * o.sk]) : 0.f;
        }
    }
    static __device__ __forceinline__ void stage(float (*s)[kT + kPad], const float* r, bool kfast) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int e = threadIdx.x + 256 * u;
            s[kfast ? e % kK : e / kT][kfast ? e / kK : e % kT] = r[u];
        }
    }
    // C tile at (i0, j0), depth [k0, k1).
    __device__ __forceinline__ void multiply(const Operand<TA>& A, const Operand<TB>& B, int i0, int j0, int k0, int k1) {
        __shared__ float sa[kK][kT + kPad], sb[kK][kT + kPad];
        const bool ka = A.sk == 1, kb = B.sk == 1;
        const int ti = threadIdx.x / 16, tj = threadIdx.x % 16;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) c[i][j] = 0.f;
        float ra[8], rb[8];
        fetch(ra, A, i0, k0, ka);
        fetch(rb, B, j0, k0, kb);
        for (int k = k0; k < k1; k += kK) {
            __syncthreads();
            stage(sa, ra, ka);
            stage(sb, rb, kb);
            __syncthreads();
            if (k + kK < k1) {
                fetch(ra, A, i0, k + kK, ka);
                fetch(rb, B, j0, k + kK, kb);
            }
#pragma unroll
            for (int kk = 0; kk < kK; ++kk) {
                float a[8], b[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 va = *reinterpret_cast<const float4*>(&sa[kk][ti * 4 + 64 * h]);
                    const float4 vb = *reinterpret_cast<const float4*>(&sb[kk][tj * 4 + 64 * h]);
                    a[4 * h] = va.x; a[4 * h + 1] = va.y; a[4 * h + 2] = va.z; a[4 * h + 3] = va.w;
                    b[4 * h] = vb.x; b[4 * h + 1] = vb.y; b[4 * h + 2] = vb.z; b[4 * h + 3] = vb.w;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) c[i][j] = fmaf(a[i], b[j], c[i][j]);
            }
        }
    }
    static __device__ __forceinline__ int row(int i) { return (threadIdx.x / 16) * 4 + (i & 3) + 64 * (i >> 2); }
    static __device__ __forceinline__ int col(int j) { return (threadIdx.x % 16) * 4 + (j & 3) + 64 * (j >> 2); }
};

// Block (row tile, segment): the segment's columns tile by tile, running
// maximum and sum per row; the 16 threads that share a row are a half warp.
template <typename T> __global__ void __launch_bounds__(256) fwd_kernel(Problem p, FwdParts parts, int tiles_per_segment) {
    const int i0 = blockIdx.x * kT, seg = blockIdx.y;
    const Operand<T> X{static_cast<const T*>(p.x), p.D, 1, p.N, p.D}, W{static_cast<const T*>(p.w), p.D, 1, p.V, p.D};
    Tile<T, T> t;
    float m[8], l[8];
    int tgt[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
        const int n = i0 + t.row(i);
        tgt[i] = n < p.N ? target_column(p, n) : kIgnored;
    }
    for (int jt = 0; jt < tiles_per_segment; ++jt) {
        const long long j0l = (long long)(seg * tiles_per_segment + jt) * kT;
        if (j0l >= p.V) break;
        const int j0 = (int)j0l;
        t.multiply(X, W, i0, j0, 0, p.D);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float mx = m[i];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int v = j0 + t.col(j);
                if (v >= p.V) t.c[i][j] = -INFINITY;
                else if (v == tgt[i]) parts.target_logit[i0 + t.row(i)] = t.c[i][j];
                mx = fmaxf(mx, t.c[i][j]);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float ms = mx == -INFINITY ? 0.f : mx;
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += expf(t.c[i][j] - ms);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            l[i] = l[i] * expf(m[i] - ms) + s;
            m[i] = mx;
        }
    }
    if (threadIdx.x % 16 == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int n = i0 + t.row(i);
            if (n < p.N) {
                parts.m[(size_t)seg * p.N + n] = m[i];
                parts.l[(size_t)seg * p.N + n] = l[i];
            }
        }
    }
}

__global__ void combine_kernel(Problem p, FwdParts parts, int segments, float* loss, float* lse) {
    grid_dependency_sync();
    const int n = blockIdx.x * blockDim.x + threadIdx.x;
    if (n >= p.N) return;
    float m = -INFINITY;
    for (int s = 0; s < segments; ++s) m = fmaxf(m, parts.m[(size_t)s * p.N + n]);
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    for (int s = 0; s < segments; ++s) l += parts.l[(size_t)s * p.N + n] * expf(parts.m[(size_t)s * p.N + n] - ms);
    const float z = m + logf(l);
    lse[n] = z;
    const int t = target_column(p, n);
    if (t == kBad) raise_status(p.status, kStatusTarget);
    loss[n] = t == kIgnored ? 0.f : t == kBad ? NAN : z - parts.target_logit[n];
}

// g[n][j] for the piece's columns; g carries dloss, so both products are plain.
template <typename T>
__global__ void __launch_bounds__(256) grad_kernel(Problem p, const float* lse, const float* dloss, float* g, int ldg, int v0,
                                                   int cols) {
    const int row_tiles = (p.N + kT - 1) / kT;
    const int i0 = (int)(blockIdx.x % row_tiles) * kT, j0 = (int)(blockIdx.x / row_tiles) * kT;
    const Operand<T> X{static_cast<const T*>(p.x), p.D, 1, p.N, p.D};
    const Operand<T> W{static_cast<const T*>(p.w) + (size_t)v0 * p.D, p.D, 1, cols, p.D};
    Tile<T, T> t;
    t.multiply(X, W, i0, j0, 0, p.D);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = i0 + t.row(i);
        if (n >= p.N) continue;
        const int tgt = target_column(p, n);
        if (tgt == kBad && v0 + j0 == 0 && t.col(0) == 0) raise_status(p.status, kStatusTarget);
        const float z = lse[n], dl = dloss[n];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = j0 + t.col(j);
            if (c >= cols) continue;
            const float e = expf(t.c[i][j] - z) - (v0 + c == tgt ? 1.f : 0.f);
            g[(size_t)n * ldg + c] = tgt < 0 ? 0.f : dl * e;
        }
    }
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }

// out[i][j] (row length ldo) = sum_k A B, plus acc[i][j] when `add`; written
// to acc as well unless `store` alone is wanted.
template <typename TA, typename TB, typename TO>
__global__ void __launch_bounds__(256) product_kernel(Operand<TA> A, Operand<TB> B, float* acc, bool add, TO* out, int ldo) {
    const int i0 = blockIdx.x * kT, j0 = blockIdx.y * kT;
    Tile<TA, TB> t;
    t.multiply(A, B, i0, j0, 0, A.depth);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i0 + t.row(i);
        if (r >= A.rows) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = j0 + t.col(j);
            if (c >= B.rows) continue;
            const size_t at = (size_t)r * ldo + c;
            const float v = t.c[i][j] + (add ? acc[at] : 0.f);
            if (out) put(out + at, v);
            else acc[at] = v;
        }
    }
}

unsigned tiles(long long n) { return (unsigned)((n + kT - 1) / kT); }

template <typename T>
cudaError_t products(const Problem& p, const float* g, int ldg, int v0, int cols, bool first, bool last, float* dx_acc, T* dx,
                     T* dw, cudaStream_t st) {
    const Operand<float> G{g, ldg, 1, p.N, cols}, Gt{g, 1, ldg, cols, p.N};
    const Operand<T> Wt{static_cast<const T*>(p.w) + (size_t)v0 * p.D, 1, p.D, p.D, cols};
    const Operand<T> Xt{static_cast<const T*>(p.x), 1, p.D, p.D, p.N};
    product_kernel<float, T, T><<<dim3(tiles(p.N), tiles(p.D)), 256, 0, st>>>(G, Wt, dx_acc, !first, last ? dx : nullptr, p.D);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    product_kernel<float, T, T><<<dim3(tiles(cols), tiles(p.D)), 256, 0, st>>>(Gt, Xt, nullptr, false, dw + (size_t)v0 * p.D, p.D);
    return cudaGetLastError();
}

}  // namespace

// Segments of the vocabulary: enough blocks for two per SM where the rows
// alone do not give them, at most 64.
int fwd_simple_segments(int N, int V) {
    const int rows = (int)tiles(N), cols = (int)tiles(V);
    return std::max(1, std::min({cols, 64, (2 * 152 + rows - 1) / std::max(rows, 1)}));
}

cudaError_t launch_fwd_simple(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st) {
    const int per = ((int)tiles(p.V) + segments - 1) / segments;
    const dim3 grid(tiles(p.N), segments);
    if (bf16) fwd_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(p, parts, per);
    else fwd_kernel<float><<<grid, 256, 0, st>>>(p, parts, per);
    return cudaGetLastError();
}

cudaError_t launch_combine(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st) {
    return launch_kernel(combine_kernel, dim3((p.N + 127) / 128), dim3(128), 0, st, p, parts, segments, loss, lse);
}

cudaError_t launch_grad_simple(const Problem& p, const float* lse, const float* dloss, float* g, int ldg, int v0, int cols,
                               bool bf16, cudaStream_t st) {
    const unsigned grid = tiles(cols) * tiles(p.N);
    if (bf16) grad_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(p, lse, dloss, g, ldg, v0, cols);
    else grad_kernel<float><<<grid, 256, 0, st>>>(p, lse, dloss, g, ldg, v0, cols);
    return cudaGetLastError();
}

cudaError_t launch_products_simple(const Problem& p, const float* g, int ldg, int v0, int cols, bool first, bool last,
                                   float* dx_acc, void* dx, void* dw, bool bf16, cudaStream_t st) {
    if (bf16) return products(p, g, ldg, v0, cols, first, last, dx_acc, (__nv_bfloat16*)dx, (__nv_bfloat16*)dw, st);
    return products(p, g, ldg, v0, cols, first, last, dx_acc, (float*)dx, (float*)dw, st);
}

}  // namespace xent
}  // namespace fibattn
