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
// Bytes of a chunk: short enough for several to a block, so that the blocks end
// together, and long enough that finding a chunk and filling its pipeline cost
// little (1.1e9 bf16 values: 1131 us with 32 KB, 1049 us with 128 KB; 6.1e7 fp32
// values: 126 us with 32 or 64 KB, 129 us with 128 KB).
constexpr int kMinChunkLog = 15, kMaxChunkLog = 18;
__host__ __device__ constexpr int chunk_values(int log, bool bf16) { return 1 << (log - (bf16 ? 1 : 2)); }
constexpr int kNormResident = 4, kClipResident = 4;   // blocks of an SM
constexpr int kBlocks = 152 * kNormResident;           // blocks (and partial sums) of a launch, at most
constexpr int kTable = 512;                // tensors of a launch, at most
constexpr int kShort = 48;                 // tensors of a short table (a launch carries its whole table)
constexpr long long kMaxBytes = 1ll << 44;   // (keeps the number of chunks within 31 bits)

struct Entry {
    const void* in;
    void* out;
    long long n;
    int first_chunk;                       // of the launch's chunks
    int bf16;
};
template <int N> struct Table {
    int entries, chunks, chunk_log;
    Entry e[N];
};

// The entry that chunk c belongs to: the last one with first_chunk <= c
// (entries without values have no chunk).
template <int N> __device__ __forceinline__ int entry_of(const Table<N>& t, int c) {
    int lo = 0, hi = t.entries - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.e[mid].first_chunk <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// A run of n values is taken in vectors of 16 bytes between its first and last
// 16-byte boundary, and value by value before and after.
template <typename T> __device__ __forceinline__ int head_of(const T* p, int n) {
    return min(n, (int)(((16u - ((unsigned)(uintptr_t)p & 15u)) & 15u) / sizeof(T)));
}

template <typename T> struct Vector {
    static constexpr int kValues = 16 / sizeof(T);
    uint4 u;
    __device__ __forceinline__ float get(int i) const {
        const unsigned* w = &u.x;
        if (sizeof(T) == 4) return __uint_as_float(w[i]);
        return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};

constexpr int kNormBatch = 8, kClipBatch = 4;   // vectors that a thread has under way at a time

// The same values as sum_squares takes with this thread, in 64 bits.
template <typename T> __device__ __noinline__ double sum_squares_wide(const T* p, int n) {
    using V = Vector<T>;
    const int head = head_of(p, n), vectors = (n - head) / V::kValues, tail = head + vectors * V::kValues;
    double s = 0.0;
    const auto add = [&](float x) { s = fma((double)x, (double)x, s); };
    if ((int)threadIdx.x < head) add(to_f(p[threadIdx.x]));
    if (tail + (int)threadIdx.x < n) add(to_f(p[tail + threadIdx.x]));
    for (int i = threadIdx.x; i < vectors; i += kThreads) {
        V v;
        v.u = __ldg(reinterpret_cast<const uint4*>(p + head) + i);
#pragma unroll
        for (int j = 0; j < V::kValues; ++j) add(v.get(j));
    }
    return s;
}

// Squares leave fp32's range long before the values do (above 1.8e19, below 1e-22).
// A thread whose sum has done so, or is so small that what was lost below 2^-149
// may count (129 terms in a run: 2^-143, 2^-33 of the limit), takes its values
// again in 64 bits; one with zeros alone does not.
constexpr float kLeastSum = 0x1p-110f;

template <typename T> __device__ __forceinline__ double sum_squares(const T* p, int n) {
    using V = Vector<T>;
    const int head = head_of(p, n), vectors = (n - head) / V::kValues, tail = head + vectors * V::kValues;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    unsigned bits = 0;                     // of all values
    if ((int)threadIdx.x < head) {         // (head and tail hold fewer than 8 values)
        const float x = to_f(p[threadIdx.x]);
        s[0] = x * x;
        bits |= __float_as_uint(x) << 1;
    }
    if (tail + (int)threadIdx.x < n) {
        const float x = to_f(p[tail + threadIdx.x]);
        s[1] = x * x;
        bits |= __float_as_uint(x) << 1;
    }
    unsigned body_bits = 0;
    const uint4* body = reinterpret_cast<const uint4*>(p + head);
    const auto add = [&](const V& v) {
        body_bits |= (v.u.x | v.u.y) | (v.u.z | v.u.w);
#pragma unroll
        for (int j = 0; j < V::kValues; ++j) {
            const float x = v.get(j);
            s[j & 3] = fmaf(x, x, s[j & 3]);
        }
    };
    int i = threadIdx.x;
    for (; i + (kNormBatch - 1) * kThreads < vectors; i += kNormBatch * kThreads) {
        V v[kNormBatch];
#pragma unroll
        for (int k = 0; k < kNormBatch; ++k) v[k].u = __ldg(body + i + k * kThreads);
#pragma unroll
        for (int k = 0; k < kNormBatch; ++k) add(v[k]);
    }
    if (i < vectors) {                     // fewer than a batch are left
        V v[kNormBatch];
#pragma unroll
        for (int k = 0; k < kNormBatch; ++k)
            v[k].u = i + k * kThreads < vectors ? __ldg(body + i + k * kThreads) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < kNormBatch; ++k) add(v[k]);
    }
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    bits |= body_bits & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu);
    if (sum >= kLeastSum && sum < INFINITY || bits == 0) return sum;
    return sum_squares_wide(p, n);
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
template <int N>
__global__ void __launch_bounds__(kThreads, kNormResident) norm_kernel(const __grid_constant__ Table<N> t, double* partial) {
    __shared__ double red[kThreads / 32];
    grid_dependency_sync();
    double s = 0.0;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const Entry& e = t.e[entry_of(t, c)];
        const long long at = (long long)(c - e.first_chunk) * chunk_values(t.chunk_log, e.bf16);
        const int n = (int)min((long long)chunk_values(t.chunk_log, e.bf16), e.n - at);
        s += e.bf16 ? sum_squares(static_cast<const __nv_bfloat16*>(e.in) + at, n)
                    : sum_squares(static_cast<const float*>(e.in) + at, n);
    }
    const double r = block_sum(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = r;
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }
__device__ __forceinline__ uint4 scaled(const Vector<float>& v, float c) {
    return make_uint4(__float_as_uint(v.get(0) * c), __float_as_uint(v.get(1) * c), __float_as_uint(v.get(2) * c),
                      __float_as_uint(v.get(3) * c));
}
__device__ __forceinline__ uint4 scaled(const Vector<__nv_bfloat16>& v, float c) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.get(2 * i) * c, v.get(2 * i + 1) * c);
        w[i] = *reinterpret_cast<const unsigned*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// (in == out is allowed: a thread reads a value before it writes it, and no other does.)
template <typename T> __device__ __forceinline__ void scale(const T* in, T* out, int n, float c) {
    using V = Vector<T>;
    const bool together = (((uintptr_t)in ^ (uintptr_t)out) & 15u) == 0;
    const int head = together ? head_of(in, n) : 0;
    const int vectors = together ? (n - head) / V::kValues : 0, tail = head + vectors * V::kValues;
    if ((int)threadIdx.x < head) put(out + threadIdx.x, to_f(in[threadIdx.x]) * c);
    const uint4* body = reinterpret_cast<const uint4*>(in + head);
    uint4* to = reinterpret_cast<uint4*>(out + head);
    int k0 = threadIdx.x;
    for (; k0 + (kClipBatch - 1) * kThreads < vectors; k0 += kClipBatch * kThreads) {
        V v[kClipBatch];
#pragma unroll
        for (int k = 0; k < kClipBatch; ++k) v[k].u = body[k0 + k * kThreads];
#pragma unroll
        for (int k = 0; k < kClipBatch; ++k) __stcs(to + k0 + k * kThreads, scaled(v[k], c));
    }
    if (k0 < vectors) {                    // fewer than a batch are left
        V v[kClipBatch];
#pragma unroll
        for (int k = 0; k < kClipBatch; ++k)
            if (k0 + k * kThreads < vectors) v[k].u = body[k0 + k * kThreads];
#pragma unroll
        for (int k = 0; k < kClipBatch; ++k)
            if (k0 + k * kThreads < vectors) __stcs(to + k0 + k * kThreads, scaled(v[k], c));
    }
    // the tail, or everything where in and out start at different offsets within 16 bytes
    for (int i = tail + threadIdx.x; i < n; i += kClipBatch * kThreads) {
        float x[kClipBatch];
#pragma unroll
        for (int k = 0; k < kClipBatch; ++k) x[k] = i + k * kThreads < n ? to_f(in[i + k * kThreads]) : 0.f;
#pragma unroll
        for (int k = 0; k < kClipBatch; ++k)
            if (i + k * kThreads < n) put(out + i + k * kThreads, x[k] * c);
    }
}

// Every block adds up all partials, in the same order, and scales its chunks.
template <int N>
__global__ void __launch_bounds__(kThreads, kClipResident) clip_kernel(const __grid_constant__ Table<N> t, const double* partial,
                                                                   int partials, float max_norm, float* norm) {
    __shared__ double red[kThreads / 32];
    grid_dependency_sync();
    double s = 0.0;
    for (int i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
    const float total = (float)sqrt(block_sum(s, red));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = total;
    // a norm that is NaN stays NaN
    const float q = max_norm / (total + 1e-6f), coef = q > 1.f ? 1.f : q;
    // from the last chunk to the first: the norm's pass read the last ones last, and L2 still holds them
    for (int c = t.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const Entry& e = t.e[entry_of(t, c)];
        if (e.out == e.in && coef == 1.f) continue;
        const long long at = (long long)(c - e.first_chunk) * chunk_values(t.chunk_log, e.bf16);
        const int n = (int)min((long long)chunk_values(t.chunk_log, e.bf16), e.n - at);
        if (e.bf16) scale(static_cast<const __nv_bfloat16*>(e.in) + at, static_cast<__nv_bfloat16*>(e.out) + at, n, coef);
        else scale(static_cast<const float*>(e.in) + at, static_cast<float*>(e.out) + at, n, coef);
    }
}

long long chunks_of(long long n, int log, bool bf16) { return (n + chunk_values(log, bf16) - 1) / chunk_values(log, bf16); }

int tables_of(int n) { return n > kTable ? (n + kTable - 1) / kTable : 1; }

template <int N>
void fill(Table<N>* t, int chunk_log, int first, int last, const void* const* grads, void* const* outs, const long long* numels,
          const int* dtypes) {
    t->entries = last - first;
    t->chunk_log = chunk_log;
    long long chunks = 0;
    for (int i = first; i < last; ++i) {
        Entry& e = t->e[i - first];
        e.in = grads[i];
        e.out = outs ? outs[i] : nullptr;
        e.n = numels[i];
        e.bf16 = dtypes[i] == FIBATTN_BF16;
        e.first_chunk = (int)chunks;
        chunks += chunks_of(numels[i], chunk_log, e.bf16);
    }
    t->chunks = (int)chunks;
}

template <typename... KArgs, typename... Args>
cudaError_t start(void (*kern)(KArgs...), int grid, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 1 : 0;
    void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};   // (the tables are not copied on the way)
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kern), at);
}

template <int N>
cudaError_t run(int n, int chunk_log, const void* const* grads, void* const* outs, const long long* numels, const int* dtypes, float max_norm,
                float* norm, double* partial, cudaStream_t st) {
    const int tables = n > N ? (n + N - 1) / N : 1;
    static thread_local Table<N> t;
    int partials = 0;
    cudaError_t e = cudaSuccess;
    for (int k = 0; k < tables && e == cudaSuccess; ++k) {
        fill(&t, chunk_log, k * N, std::min(n, (k + 1) * N), grads, outs, numels, dtypes);
        const int grid = std::max(1, std::min(kBlocks, t.chunks));
        ProfScope s("grad_norm", st);
        e = start(norm_kernel<N>, grid, st, t, partial + partials);
        partials += grid;
    }
    for (int k = 0; k < (outs ? tables : 1) && e == cudaSuccess; ++k) {
        if (tables > 1) fill(&t, chunk_log, k * N, std::min(n, (k + 1) * N), grads, outs, numels, dtypes);
        if (!outs) t.chunks = 0;                 // the norm alone
        const int grid = std::max(1, std::min(152 * kClipResident, t.chunks));
        ProfScope s("grad_clip", st);
        e = start(clip_kernel<N>, grid, st, t, static_cast<const double*>(partial), partials, max_norm,
                  k == 0 ? norm : static_cast<float*>(nullptr));
    }
    return e;
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
    long long bytes = 0;
    for (int i = 0; i < n; ++i) {
        if (dtypes[i] != FIBATTN_F32 && dtypes[i] != FIBATTN_BF16)
            return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: unknown dtype %d", i, dtypes[i]);
        if (numels[i] < 0) return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: negative size", i);
        if (numels[i] && (!grads[i] || (outs && !outs[i])))
            return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: NULL pointer", i);
        const uintptr_t es = dtypes[i] == FIBATTN_BF16 ? 2 : 4;
        if (((uintptr_t)grads[i] | (outs ? (uintptr_t)outs[i] : 0)) & (es - 1))
            return set_errorf(FIBATTN_ERR_INVALID_ARG, "tensor %d: pointer not aligned to its element", i);
        if (numels[i] > kMaxBytes || (bytes += numels[i] * (long long)es) > kMaxBytes)
            return set_error(FIBATTN_ERR_INVALID_ARG, "too many values");
    }
    int rc = bind_device_context();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    int chunk_log = kMinChunkLog;              // six chunks or more to a block
    while (chunk_log < kMaxChunkLog && (bytes >> (chunk_log + 1)) >= 6ll * kBlocks) ++chunk_log;
    const cudaError_t e = n <= kShort ? run<kShort>(n, chunk_log, grads, outs, numels, dtypes, max_norm, norm, partial, st)
                                      : run<kTable>(n, chunk_log, grads, outs, numels, dtypes, max_norm, norm, partial, st);
    if (e != cudaSuccess) return set_errorf(FIBATTN_ERR_CUDA, "gradient clipping launch: %s", cudaGetErrorString(e));
    return FIBATTN_OK;
}

}  // extern "C"
