// xent_rows.cu -- the cross entropy's forward for few rows (a decoding step's
// tokens), and the join of per-row statistics.
//
// With few rows the work is one pass over w, so this kernel is built as a
// stream: every warp takes a run of consecutive rows of w, four at a time, a
// lane 16 bytes of each per step, against x in shared memory (fp32).  Products
// and sums are fp32 FMAs for either type.  Bound by memory.
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
    for (int o = 16 / K; o > 0; o /= 2) r += __shfl_xor_sync(0xffffffffu, r, o);
    return r;
}

// VECTORS: rows start on 16-byte boundaries.
template <typename T, int NT, bool VECTORS>
__global__ void __launch_bounds__(32 * kWarps) rows_kernel(Problem p, FwdParts parts, int segments) {
    extern __shared__ float xs[];                  // [NT][steps * 256]
    __shared__ float red_m[kWarps][NT], red_l[kWarps][NT];
    constexpr int kValues = NT * kGroup;           // logits of a group of rows of w, value n * kGroup + r
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n0 = blockIdx.y * NT, steps = (p.D + 255) / 256;
    grid_dependency_sync();
    for (int i = threadIdx.x; i < NT * steps * 256; i += 32 * kWarps) {
        const int n = i / (steps * 256), k = i % (steps * 256);
        const bool in = n0 + n < p.N && k < p.D;
        xs[n * steps * 256 + (VECTORS ? staged(k) : k)] =
            in ? to_f(static_cast<const T*>(p.x)[(size_t)(n0 + n) * p.D + k]) : 0.f;
    }
    // a lane keeps the statistics of the logits that the reduction leaves with it: row n0 + n, every kGroup-th column
    const int own = lane / (32 / kValues), own_n = own / kGroup, own_r = own % kGroup;
    const bool writes = lane % (32 / kValues) == 0;
    const int target = n0 + own_n < p.N ? target_column(p, n0 + own_n) : kIgnored;
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
                for (int r = 0; r < kGroup; ++r) {
                    if (k < p.D && v0 + r < hi) {
                        Vec8<T>::load(w + (size_t)(v0 + r) * p.D + k, a[r]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) a[r][j] = 0.f;
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float* q = xs + (n * steps + st) * 256 + lane * 4;
                    const float4 q0 = *reinterpret_cast<const float4*>(q), q1 = *reinterpret_cast<const float4*>(q + 128);
#pragma unroll
                    for (int r = 0; r < kGroup; ++r) {
                        s[n * kGroup + r] = fmaf(a[r][0], q0.x, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][1], q0.y, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][2], q0.z, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][3], q0.w, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][4], q1.x, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][5], q1.y, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][6], q1.z, s[n * kGroup + r]);
                        s[n * kGroup + r] = fmaf(a[r][7], q1.w, s[n * kGroup + r]);
                    }
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
            if (v0 + own_r == target && writes) parts.target_logit[n0 + own_n] = mine;
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
    if (threadIdx.x < NT && n0 + (int)threadIdx.x < p.N) {
        const int n = threadIdx.x;
        float top = -INFINITY, sum = 0.f;
        for (int w8 = 0; w8 < kWarps; ++w8) top = fmaxf(top, red_m[w8][n]);
        const float ms = top == -INFINITY ? 0.f : top;
        for (int w8 = 0; w8 < kWarps; ++w8) sum += red_l[w8][n] * expf(red_m[w8][n] - ms);
        parts.m[(size_t)(n0 + n) * segments + blockIdx.x] = top;
        parts.l[(size_t)(n0 + n) * segments + blockIdx.x] = sum;
    }
}

__device__ __forceinline__ void finish_row(const Problem& p, const FwdParts& parts, int n, float z, float* loss, float* lse) {
    lse[n] = z;
    const int t = target_column(p, n);
    if (t == kBad) raise_status(p.status, kStatusTarget);
    loss[n] = t == kIgnored ? 0.f : t == kBad ? NAN : z - parts.target_logit[n];
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

template <typename T, int NT> cudaError_t launch_rows(const Problem& p, const FwdParts& parts, int segments, cudaStream_t st) {
    const size_t smem = (size_t)NT * ((p.D + 255) / 256) * 256 * 4;
    const dim3 grid(segments, (p.N + NT - 1) / NT);
    if (p.D % (16 / sizeof(T)) == 0 && p.D % 8 == 0)
        return launch_kernel(rows_kernel<T, NT, true>, grid, dim3(32 * kWarps), smem, st, p, parts, segments);
    return launch_kernel(rows_kernel<T, NT, false>, grid, dim3(32 * kWarps), smem, st, p, parts, segments);
}

// Rows of x that a block takes: as many as there are, up to eight, and as fit
// 47 KB of shared memory (w is read again, from L2, for each further group).
template <typename T> cudaError_t rows(const Problem& p, const FwdParts& parts, int segments, cudaStream_t st) {
    int nt = p.N <= 1 ? 1 : p.N <= 2 ? 2 : p.N <= 4 ? 4 : 8;
    while (nt > 1 && nt * ((p.D + 255) / 256) > 47) nt /= 2;
    switch (nt) {
    case 1: return launch_rows<T, 1>(p, parts, segments, st);
    case 2: return launch_rows<T, 2>(p, parts, segments, st);
    case 4: return launch_rows<T, 4>(p, parts, segments, st);
    default: return launch_rows<T, 8>(p, parts, segments, st);
    }
}

}  // namespace

int few_rows_segments(int N, int V) {
    return std::max(1, std::min(152 * 4, (V + kGroup * kWarps - 1) / (kGroup * kWarps)));
}

cudaError_t launch_few_rows(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st) {
    return bf16 ? rows<__nv_bfloat16>(p, parts, segments, st) : rows<float>(p, parts, segments, st);
}

cudaError_t launch_join_segments(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st) {
    return launch_kernel(join_segments_kernel, dim3((p.N + 31) / 32), dim3(256), 0, st, p, parts, segments, loss, lse);
}

cudaError_t launch_join_rows(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st) {
    return launch_kernel(join_rows_kernel, dim3(p.N), dim3(256), 0, st, p, parts, segments, loss, lse);
}

}  // namespace xent
}  // namespace fibattn
