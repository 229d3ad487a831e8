// grad_clip.cu -- global gradient norm over many tensors, and clipping
// (include/fibattn.h, fibattn_clip_grads).
//
//   norm = sqrt(sum of squares),  out = grad * min(1, max_norm / (norm + 1e-6)).
//
// Bound by memory: every value is read for the norm, read again to be scaled
// and written.  The tensors travel as a table in the launch parameters (no
// copy to the device), cut into chunks that the blocks take in turn.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/fibattn.h"
#include "fibattn_internal.cuh"

using namespace fibattn;

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16384;              // values of a chunk: 64 of each thread
constexpr int kBlocks = 152 * 4;           // blocks of a launch, at most
constexpr int kTable = 512;                // tensors of a launch, at most
constexpr long long kMaxChunks = 1ll << 30;

struct Entry {
    const void* in;
    void* out;
    long long n;
    int first_chunk;                       // of the launch's chunks
    int bf16;
};
struct Table {
    int entries, chunks;
    Entry e[kTable];
};

// The entry that chunk c belongs to: the last one with first_chunk <= c
// (entries without values have no chunk).
__device__ __forceinline__ int entry_of(const Table& t, int c) {
    int lo = 0, hi = t.entries - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.e[mid].first_chunk <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <typename T> __device__ __forceinline__ float sum_squares(const T* p, int n) {
    float s = 0.f;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const float x = to_f(p[i]);
        s = fmaf(x, x, s);
    }
    return s;
}

__device__ double block_sum(double s, double* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = s;
    __syncthreads();
    double r = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) r += red[w];
    return r;
}

// partial[b]: block b's sum of squares over its chunks b, b + gridDim, ...
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Table t, double* partial) {
    __shared__ double red[kThreads / 32];
    grid_dependency_sync();
    double s = 0.0;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const Entry& e = t.e[entry_of(t, c)];
        const long long at = (long long)(c - e.first_chunk) * kChunk;
        const int n = (int)min((long long)kChunk, e.n - at);
        s += e.bf16 ? sum_squares(static_cast<const __nv_bfloat16*>(e.in) + at, n)
                    : sum_squares(static_cast<const float*>(e.in) + at, n);
    }
    const double r = block_sum(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = r;
}

__device__ __forceinline__ void scale(const float* in, float* out, int n, float c) {
    for (int i = threadIdx.x; i < n; i += kThreads) out[i] = in[i] * c;
}
__device__ __forceinline__ void scale(const __nv_bfloat16* in, __nv_bfloat16* out, int n, float c) {
    for (int i = threadIdx.x; i < n; i += kThreads) out[i] = __float2bfloat16(to_f(in[i]) * c);
}

// Every block adds up all partials, in the same order, and scales its chunks.
__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ Table t, const double* partial, int partials,
                                                        float max_norm, float* norm) {
    __shared__ double red[kThreads / 32];
    grid_dependency_sync();
    double s = 0.0;
    for (int i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
    const float total = (float)sqrt(block_sum(s, red));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = total;
    // a norm that is NaN stays NaN
    const float q = max_norm / (total + 1e-6f), coef = q > 1.f ? 1.f : q;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const Entry& e = t.e[entry_of(t, c)];
        if (e.out == e.in && coef == 1.f) continue;
        const long long at = (long long)(c - e.first_chunk) * kChunk;
        const int n = (int)min((long long)kChunk, e.n - at);
        if (e.bf16) scale(static_cast<const __nv_bfloat16*>(e.in) + at, static_cast<__nv_bfloat16*>(e.out) + at, n, coef);
        else scale(static_cast<const float*>(e.in) + at, static_cast<float*>(e.out) + at, n, coef);
    }
}

int tables_of(int n) { return n > kTable ? (n + kTable - 1) / kTable : 1; }

void fill(Table* t, int first, int last, const void* const* grads, void* const* outs, const long long* numels,
          const int* dtypes) {
    t->entries = last - first;
    long long chunks = 0;
    for (int i = first; i < last; ++i) {
        Entry& e = t->e[i - first];
        e.in = grads[i];
        e.out = outs ? outs[i] : nullptr;
        e.n = numels[i];
        e.bf16 = dtypes[i] == FIBATTN_BF16;
        e.first_chunk = (int)chunks;
        chunks += (numels[i] + kChunk - 1) / kChunk;
    }
    t->chunks = (int)chunks;
}

}  // namespace

extern "C" {

size_t fibattn_clip_grads_workspace_bytes(int n) {
    if (n < 0 || n > (1 << 20)) {
        set_errorf(FIBATTN_ERR_INVALID_ARG, "n must be in [0, 2^20] (got %d)", n);
        return 0;
    }
    return (size_t)tables_of(n) * kBlocks * sizeof(double);
}

int fibattn_clip_grads(int n, const void* const* grads, void* const* outs, const long long* numels, const int* dtypes,
                       float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    if (n < 0 || n > (1 << 20)) return set_errorf(FIBATTN_ERR_INVALID_ARG, "n must be in [0, 2^20] (got %d)", n);
    if (n > 0 && (!grads || !numels || !dtypes)) return set_error(FIBATTN_ERR_INVALID_ARG, "NULL array");
    if (!norm || !workspace) return set_error(FIBATTN_ERR_INVALID_ARG, "NULL norm or workspace pointer");
    if (((uintptr_t)norm & 3u) || ((uintptr_t)workspace & 15u))
        return set_error(FIBATTN_ERR_INVALID_ARG, "workspace must be 16-byte aligned (norm: 4-byte)");
    if (!(max_norm >= 0.f)) return set_errorf(FIBATTN_ERR_INVALID_ARG, "max_norm must be >= 0 (got %g)", (double)max_norm);
    if (workspace_bytes < fibattn_clip_grads_workspace_bytes(n))
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "workspace too small: %zu < %zu", workspace_bytes,
                          fibattn_clip_grads_workspace_bytes(n));
    long long chunks = 0;
    for (int i = 0; i < n; ++i) {
        if (dtypes[i] != FIBATTN_F32 && dtypes[i] != FIBATTN_BF16)
            return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: unknown dtype %d", i, dtypes[i]);
        if (numels[i] < 0) return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: negative size", i);
        if (numels[i] && (!grads[i] || (outs && !outs[i])))
            return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: NULL pointer", i);
        const uintptr_t es = dtypes[i] == FIBATTN_BF16 ? 2 : 4;
        if (((uintptr_t)grads[i] | (outs ? (uintptr_t)outs[i] : 0)) & (es - 1))
            return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: pointer not aligned to its element", i);
        if (numels[i] > kMaxChunks * kChunk || (chunks += (numels[i] + kChunk - 1) / kChunk) > kMaxChunks)
            return set_error(FIBATTN_ERR_INVALID_ARG, "too many values");
    }
    int rc = bind_device_context();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    const int tables = tables_of(n);
    int partials = 0;
    static thread_local Table t;
    cudaError_t e = cudaSuccess;
    for (int k = 0; k < tables && e == cudaSuccess; ++k) {
        fill(&t, k * kTable, std::min(n, (k + 1) * kTable), grads, outs, numels, dtypes);
        const int grid = std::max(1, std::min(kBlocks, t.chunks));
        ProfScope s("grad_norm", st);
        e = launch_kernel(norm_kernel, dim3(grid), dim3(kThreads), 0, st, t, partial + partials);
        partials += grid;
    }
    for (int k = 0; k < tables && e == cudaSuccess; ++k) {
        fill(&t, k * kTable, std::min(n, (k + 1) * kTable), grads, outs, numels, dtypes);
        const int grid = outs ? std::max(1, std::min(kBlocks, t.chunks)) : 1;
        if (!outs) t.chunks = 0;
        ProfScope s("grad_clip", st);
        e = launch_kernel(clip_kernel, dim3(grid), dim3(kThreads), 0, st, t, partial, partials, max_norm, k == 0 ? norm : nullptr);
        if (!outs) break;
    }
    if (e != cudaSuccess) return set_errorf(FIBATTN_ERR_CUDA, "gradient clipping launch: %s", cudaGetErrorString(e));
    return FIBATTN_OK;
}

}  // extern "C"
