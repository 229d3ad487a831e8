// xent_stream.cu -- the cross entropy for one to four rows (a decoding step's
// tokens): one stream over w on the fp32 pipes.
//
// Every warp takes a run of consecutive rows of w, four at a time, a lane 16 bytes
// of each per step, against x in shared memory (fp32).  The gradient is one pass
// too: the logits, g and both products of a batch of rows of w while it is in
// cache.  Bound by memory for one row, by the FMA rate and the reductions from
// about four, which come here only over small heads (us on the GPU forward +
// backward, 512 wide, bf16: one row over 32768 columns 8.9 + 24.2, w being read in
// 5.0 at the peak; four over 4000 columns 6.2 + 11.2).
#include <algorithm>

#include "xent.cuh"

namespace fibattn {
namespace xent {
namespace {

constexpr int kWarps = 8;
constexpr int kGroup = 4;                          // rows of w that a warp has under way

// x of one step of a row (256 values: 8 per lane) is laid out as the lanes'
// first four values, then their last four, so that a warp's 16-byte reads touch
// every bank once.
__device__ __forceinline__ int staged(int k) { return (k & ~255) + ((k >> 2) & 1) * 128 + ((k >> 3) & 31) * 4 + (k & 3); }

// s[i] summed over the warp, one value to each lane: returns the sum of value
// owner(lane) = lane / (32 / K).  Halving exchanges: K - 1 shuffles and one for
// each bit that is left, where a butterfly for every value would take 5 K.
template <int K> __device__ __forceinline__ float sum_to_owner(float* s, int lane) {
#pragma unroll
    for (int h = K / 2, o = 16; h > 0; h /= 2, o /= 2) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float give = up ? s[i] : s[i + h], keep = up ? s[i + h] : s[i];
            s[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    float r = s[0];
#pragma unroll
    for (int o = 1; o < 32 / K; o *= 2) r += __shfl_xor_sync(0xffffffffu, r, o);
    return r;
}

// Eight values at p, of which `n` are there (zeros, or no write, past them).
// VECTORS: rows start on 16-byte boundaries and n is 0 or less, or 8 or more.
template <typename T, bool VECTORS> __device__ __forceinline__ void load8(const T* p, int n, float* x) {
    if (VECTORS && n > 0) {
        Vec8<T>::load(p, x);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = !VECTORS && j < n ? to_f(p[j]) : 0.f;
}
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }
template <typename T, bool VECTORS> __device__ __forceinline__ void store8(T* p, int n, const float* x) {
    if constexpr (VECTORS) {
        if (n > 0) Vec8<T>::store(p, x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) put(p + j, x[j]);
    }
}
__device__ __forceinline__ float dot8(const float* a, const float4& q0, const float4& q1, float s) {
    s = fmaf(a[0], q0.x, s); s = fmaf(a[1], q0.y, s); s = fmaf(a[2], q0.z, s); s = fmaf(a[3], q0.w, s);
    s = fmaf(a[4], q1.x, s); s = fmaf(a[5], q1.y, s); s = fmaf(a[6], q1.z, s); return fmaf(a[7], q1.w, s);
}
// Value j of thread t in an array of eight for each of 256 threads.
__device__ __forceinline__ float& red_at(float* s, int t, int j) { return s[j * 32 * kWarps + t]; }

template <typename T, int NT, bool VECTORS>
__global__ void __launch_bounds__(32 * kWarps) stream_kernel(Problem p, FwdParts parts, int segments) {
    extern __shared__ float xs[];                  // [NT][steps * 256]
    __shared__ float red_m[kWarps][NT], red_l[kWarps][NT];
    constexpr int kValues = NT * kGroup;           // logits of a group of rows of w, value n * kGroup + r
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int steps = (p.D + 255) / 256;
    grid_dependency_sync();
    for (int i = threadIdx.x; i < NT * steps * 256; i += 32 * kWarps) {
        const int n = i / (steps * 256), k = i % (steps * 256);
        const bool in = n < p.N && k < p.D;
        xs[n * steps * 256 + (VECTORS ? staged(k) : k)] =
            in ? to_f(static_cast<const T*>(p.x)[(size_t)n * p.D + k]) : 0.f;
    }
    // a lane keeps the statistics of the logits that the reduction leaves with it: row n, every kGroup-th column
    const int own = lane / (32 / kValues), own_n = own / kGroup, own_r = own % kGroup;
    const bool writes = lane % (32 / kValues) == 0;
    const int target = own_n < p.N ? target_column(p, own_n) : kIgnored;
    float m = -INFINITY, l = 0.f;
    __syncthreads();
    const int worker = blockIdx.x * kWarps + warp, workers = gridDim.x * kWarps;
    const int lo = (int)((long long)p.V * worker / workers), hi = (int)((long long)p.V * (worker + 1) / workers);
    const T* w = static_cast<const T*>(p.w);
    for (int v0 = lo; v0 < hi; v0 += kGroup) {
        float s[kValues];
#pragma unroll
        for (int i = 0; i < kValues; ++i) s[i] = 0.f;
        if (VECTORS) {
#pragma unroll 2
            for (int st = 0; st < steps; ++st) {
                const int k = st * 256 + lane * 8;
                float a[kGroup][8];
#pragma unroll
                for (int r = 0; r < kGroup; ++r) load8<T, true>(w + (size_t)(v0 + r) * p.D + k, v0 + r < hi ? p.D - k : 0, a[r]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float* q = xs + (n * steps + st) * 256 + lane * 4;
                    const float4 q0 = *reinterpret_cast<const float4*>(q), q1 = *reinterpret_cast<const float4*>(q + 128);
#pragma unroll
                    for (int r = 0; r < kGroup; ++r) s[n * kGroup + r] = dot8(a[r], q0, q1, s[n * kGroup + r]);
                }
            }
        } else {
#pragma unroll 2
            for (int k = lane; k < p.D; k += 32) {
                float a[kGroup];
#pragma unroll
                for (int r = 0; r < kGroup; ++r) a[r] = v0 + r < hi ? to_f(w[(size_t)(v0 + r) * p.D + k]) : 0.f;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float q = xs[n * steps * 256 + k];
#pragma unroll
                    for (int r = 0; r < kGroup; ++r) s[n * kGroup + r] = fmaf(a[r], q, s[n * kGroup + r]);
                }
            }
        }
        const float mine = sum_to_owner<kValues>(s, lane);
        if (v0 + own_r < hi) {
            if (v0 + own_r == target && writes) parts.target_logit[own_n] = mine;
            const float top = fmaxf(m, mine), ms = top == -INFINITY ? 0.f : top;
            l = l * expf(m - ms) + expf(mine - ms);
            m = top;
        }
    }
    // the kGroup owners of a row of x: neighbours of 32 / kValues lanes each
#pragma unroll
    for (int o = 32 / kValues; o < 32 / NT; o *= 2) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
        const float top = fmaxf(m, m2), ms = top == -INFINITY ? 0.f : top;
        l = l * expf(m - ms) + l2 * expf(m2 - ms);
        m = top;
    }
    if (writes && own_r == 0) {
        red_m[warp][own_n] = m;
        red_l[warp][own_n] = l;
    }
    __syncthreads();
    if (threadIdx.x < NT && (int)threadIdx.x < p.N) {
        const int n = threadIdx.x;
        float top = -INFINITY, sum = 0.f;
        for (int w8 = 0; w8 < kWarps; ++w8) top = fmaxf(top, red_m[w8][n]);
        const float ms = top == -INFINITY ? 0.f : top;
        for (int w8 = 0; w8 < kWarps; ++w8) sum += red_l[w8][n] * expf(red_m[w8][n] - ms);
        parts.m[(size_t)n * segments + blockIdx.x] = top;
        parts.l[(size_t)n * segments + blockIdx.x] = sum;
    }
}

// The gradient of few rows in one pass over w: a block forms the logits of a
// batch of 32 rows of w as stream_kernel does, turns them into g in shared memory,
// and then takes the batch again (from L1) with a thread for eight columns:
//   dw[v] = sum_n g[n][v] x[n]   to memory,   dx[n] += g[n][v] w[v]   in registers.
// parts[block][n][D]: dx over the block's rows of w.
template <typename T, int NT, bool VECTORS>
__global__ void __launch_bounds__(32 * kWarps) stream_gradient_kernel(Problem p, const float* lse, const float* dloss, T* dw, float* parts,
                                                                    bool want_dx) {
    extern __shared__ float xs[];                  // [NT][steps * 256], staged
    constexpr int kValues = NT * kGroup, kBatch = kGroup * kWarps;
    __shared__ float gs[kBatch][NT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, steps = (p.D + 255) / 256;
    grid_dependency_sync();
    for (int i = threadIdx.x; i < NT * steps * 256; i += 32 * kWarps) {
        const int n = i / (steps * 256), k = i % (steps * 256);
        xs[n * steps * 256 + staged(k)] = n < p.N && k < p.D ? to_f(static_cast<const T*>(p.x)[(size_t)n * p.D + k]) : 0.f;
    }
    const int own = lane / (32 / kValues), own_n = own / kGroup, own_r = own % kGroup;
    const bool writes = lane % (32 / kValues) == 0;
    const int target = own_n < p.N ? target_column(p, own_n) : kIgnored;
    const float z = target >= 0 ? lse[own_n] : 0.f, dl = target >= 0 ? dloss[own_n] : 0.f;
    if (target == kBad && blockIdx.x == 0 && writes && own_r == 0) raise_status(p.status, kStatusTarget);
    // columns 8 cg .. of the rows rg, rg + groups, ... of a batch
    const int column_groups = (p.D + 7) / 8, groups = 32 * kWarps / column_groups;
    const int cg = threadIdx.x % column_groups, rg = threadIdx.x / column_groups;
    const bool takes = rg < groups;
    const int at = (cg >> 5) * 256 + (cg & 31) * 4;           // staged(8 cg)
    float dx[NT][8];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) dx[n][j] = 0.f;
    const int lo = (int)((long long)p.V * blockIdx.x / gridDim.x), hi = (int)((long long)p.V * (blockIdx.x + 1) / gridDim.x);
    const T* w = static_cast<const T*>(p.w);
    for (int b0 = lo; b0 < hi; b0 += kBatch) {
        __syncthreads();                           // x is staged; the batch before has been read
        const int v0 = b0 + warp * kGroup;
        float s[kValues];
#pragma unroll
        for (int i = 0; i < kValues; ++i) s[i] = 0.f;
        if (v0 < hi) {
#pragma unroll 2
            for (int st = 0; st < steps; ++st) {
                const int k = st * 256 + lane * 8;
                float a[kGroup][8];
#pragma unroll
                for (int r = 0; r < kGroup; ++r) load8<T, VECTORS>(w + (size_t)(v0 + r) * p.D + k, v0 + r < hi ? p.D - k : 0, a[r]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float* q = xs + (n * steps + st) * 256 + lane * 4;
                    const float4 q0 = *reinterpret_cast<const float4*>(q), q1 = *reinterpret_cast<const float4*>(q + 128);
#pragma unroll
                    for (int r = 0; r < kGroup; ++r) s[n * kGroup + r] = dot8(a[r], q0, q1, s[n * kGroup + r]);
                }
            }
        }
        const float mine = sum_to_owner<kValues>(s, lane);
        if (writes) gs[warp * kGroup + own_r][own_n] = target < 0 ? 0.f : dl * (expf(mine - z) - (v0 + own_r == target ? 1.f : 0.f));
        __syncthreads();
        const int rows = min(kBatch, hi - b0);
        if (takes) {
            for (int r = rg; r < rows; r += groups) {
                float a[8], o[8];
                load8<T, VECTORS>(w + (size_t)(b0 + r) * p.D + 8 * cg, p.D - 8 * cg, a);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = 0.f;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float g = gs[r][n];
                    const float* q = xs + n * steps * 256 + at;
                    const float4 q0 = *reinterpret_cast<const float4*>(q), q1 = *reinterpret_cast<const float4*>(q + 128);
                    o[0] = fmaf(g, q0.x, o[0]); o[1] = fmaf(g, q0.y, o[1]); o[2] = fmaf(g, q0.z, o[2]); o[3] = fmaf(g, q0.w, o[3]);
                    o[4] = fmaf(g, q1.x, o[4]); o[5] = fmaf(g, q1.y, o[5]); o[6] = fmaf(g, q1.z, o[6]); o[7] = fmaf(g, q1.w, o[7]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dx[n][j] = fmaf(g, a[j], dx[n][j]);
                }
                if (dw) store8<T, VECTORS>(dw + (size_t)(b0 + r) * p.D + 8 * cg, p.D - 8 * cg, o);
            }
        }
    }
    if (!want_dx) return;
    // the groups' sums of a column, one row of x at a time, over the space of x
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();
        if (takes)
#pragma unroll
            for (int j = 0; j < 8; ++j) red_at(xs, rg * column_groups + cg, j) = dx[n][j];
        __syncthreads();
        for (int o = threadIdx.x; n < p.N && o < 8 * column_groups; o += 32 * kWarps) {
            const int c = o % column_groups, j = o / column_groups;
            float sum = 0.f;
            for (int i = 0; i < groups; ++i) sum += red_at(xs, i * column_groups + c, j);
            if (8 * c + j < p.D) parts[((size_t)blockIdx.x * p.N + n) * p.D + 8 * c + j] = sum;
        }
    }
}

template <typename T, int NT> cudaError_t launch_rows(const Problem& p, const FwdParts& parts, int segments, cudaStream_t st) {
    const size_t smem = (size_t)NT * ((p.D + 255) / 256) * 256 * 4;
    const dim3 grid(segments);
    if (p.D % (16 / sizeof(T)) == 0 && p.D % 8 == 0)
        return launch_kernel(stream_kernel<T, NT, true>, grid, dim3(32 * kWarps), smem, st, p, parts, segments);
    return launch_kernel(stream_kernel<T, NT, false>, grid, dim3(32 * kWarps), smem, st, p, parts, segments);
}

template <typename T> cudaError_t rows(const Problem& p, const FwdParts& parts, int segments, cudaStream_t st) {
    if (p.N == 1) return launch_rows<T, 1>(p, parts, segments, st);
    return p.N == 2 ? launch_rows<T, 2>(p, parts, segments, st) : launch_rows<T, 4>(p, parts, segments, st);
}

template <typename T, int NT>
cudaError_t launch_rows_gradient(const Problem& p, const float* lse, const float* dloss, void* dw, float* parts, bool want_dx,
                                 int blocks, cudaStream_t st) {
    // x, and later eight values of each of the block's threads
    const size_t smem = std::max((size_t)NT * ((p.D + 255) / 256) * 256 * 4, (size_t)32 * kWarps * 8 * 4);
    if (p.D % 8 == 0)
        return launch_kernel(stream_gradient_kernel<T, NT, true>, dim3(blocks), dim3(32 * kWarps), smem, st, p, lse, dloss,
                             static_cast<T*>(dw), parts, want_dx);
    return launch_kernel(stream_gradient_kernel<T, NT, false>, dim3(blocks), dim3(32 * kWarps), smem, st, p, lse, dloss,
                         static_cast<T*>(dw), parts, want_dx);
}
template <typename T>
cudaError_t rows_gradient(const Problem& p, const float* lse, const float* dloss, void* dx, void* dw, float* parts, int blocks,
                          cudaStream_t st) {
    cudaError_t e;
    {
        ProfScope s("xent_stream_grad", st);
        const bool want_dx = dx != nullptr;
        e = p.N == 1   ? launch_rows_gradient<T, 1>(p, lse, dloss, dw, parts, want_dx, blocks, st)
            : p.N == 2 ? launch_rows_gradient<T, 2>(p, lse, dloss, dw, parts, want_dx, blocks, st)
                       : launch_rows_gradient<T, 4>(p, lse, dloss, dw, parts, want_dx, blocks, st);
    }
    return e != cudaSuccess || !dx ? e : launch_join_dx(p, parts, blocks, dx, sizeof(T) == 2, st);
}

}  // namespace

bool stream_applies(int N, int D) { return N <= 4 && D <= 2048; }

int stream_segments(int V) { return std::max(1, std::min(152 * 4, (V + kGroup * kWarps - 1) / (kGroup * kWarps))); }

cudaError_t launch_stream(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st) {
    return bf16 ? rows<__nv_bfloat16>(p, parts, segments, st) : rows<float>(p, parts, segments, st);
}

int stream_blocks(int V) { return std::max(1, std::min(152 * 2, (V + kGroup * kWarps - 1) / (kGroup * kWarps))); }

cudaError_t launch_stream_gradient(const Problem& p, const float* lse, const float* dloss, void* dx, void* dw, float* parts, int blocks,
                                   bool bf16, cudaStream_t st) {
    return bf16 ? rows_gradient<__nv_bfloat16>(p, lse, dloss, dx, dw, parts, blocks, st)
                : rows_gradient<float>(p, lse, dloss, dx, dw, parts, blocks, st);
}

}  // namespace xent
}  // namespace fibattn
