// cache_append.cu -- keys and values of new tokens into a paged cache, the keys
// rotated on the way: k~ = R(pos) k (arXiv 2606.28560, Section 2: RoPE at true
// positions, before the gather), values as they are.
#include <algorithm>

#include "cache.cuh"

namespace fibattn {
namespace cache {

namespace {

template <typename T>
__device__ __forceinline__ void copy_chunk(const T* from, T* to, int c) {
    constexpr int n = (int)sizeof(T) / 2;            // 16-byte vectors in 8 elements
    const uint4* f = reinterpret_cast<const uint4*>(from + 8 * c);
    const uint4* g = reinterpret_cast<const uint4*>(from + kHalf + 8 * c);
    uint4 x[2 * n];
#pragma unroll
    for (int i = 0; i < n; ++i) { x[i] = f[i]; x[n + i] = g[i]; }
#pragma unroll
    for (int i = 0; i < n; ++i) {
        reinterpret_cast<uint4*>(to + 8 * c)[i] = x[i];
        reinterpret_cast<uint4*>(to + kHalf + 8 * c)[i] = x[n + i];
    }
}

// A thread has a token's pairs 8c .. 8c+7 for a run of heads: the angles are
// evaluated once for the run.  Bound by memory: each value is read and written once.
template <typename T>
__global__ void __launch_bounds__(256) append_kernel(const __grid_constant__ AppendArgs a) {
    using R = typename RotOf<T>::type;
    grid_dependency_sync();
    const int runs = (a.c.Hkv + a.heads - 1) / a.heads;
    const long long items = (long long)a.N * runs * 4;
    const long long it = blockIdx.x * (long long)blockDim.x + threadIdx.x;
    if (it >= items) return;
    const int c = (int)(it & 3), run = (int)((it >> 2) % runs), n = (int)((it >> 2) / runs);
    const int pos = a.positions[n], seq = a.seqs ? a.seqs[n] : n;
    if (pos < 0 || seq < 0) return;                  // padding
    unsigned row = 0;
    const int slot = a.slots ? a.slots[n] : pos;
    if (seq >= a.c.seqs || !locate(a.c, a.c.table + (size_t)seq * a.c.pages_per_seq, slot, row)) {
        raise_status(a.status, kStatusPage);
        return;
    }
    float cs[8], sn[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) rope_cs_f32(a.c.rope, 8 * c + u, pos, cs[u], sn[u]);
    float largest = 0.f;
    const int h1 = min(a.c.Hkv, (run + 1) * a.heads);
    for (int h = run * a.heads; h < h1; ++h) {
        const size_t at = (size_t)(row + h * a.c.head_stride) * kHeadDim;
        float x[16];
        load_chunk(static_cast<const T*>(a.k) + n * a.k_token + h * a.k_head, c, x);
        copy_chunk(static_cast<const T*>(a.v) + n * a.v_token + h * a.v_head, static_cast<T*>(a.c.v) + at, c);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float p = x[u], q = x[8 + u];
            x[u] = p * cs[u] - q * sn[u];
            x[8 + u] = q * cs[u] + p * sn[u];
            largest = fmaxf(largest, fmaxf(fabsf(x[u]), fabsf(x[8 + u])));
        }
        store_chunk(static_cast<R*>(a.c.k) + at, c, x);
    }
    if (sizeof(R) == 2 && largest >= 65520.f) raise_status(a.status, kStatusRange);   // rounds to infinity in fp16
}

}  // namespace

cudaError_t launch_append(const AppendArgs& args, bool bf16, cudaStream_t st) {
    AppendArgs a = args;
    a.heads = (long long)a.N * a.c.Hkv * 4 > 152 * 2048 ? a.c.Hkv : 1;
    const long long items = (long long)a.N * ((a.c.Hkv + a.heads - 1) / a.heads) * 4;
    const dim3 grid((unsigned)((items + 255) / 256));
    return bf16 ? launch_kernel(append_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, a)
                : launch_kernel(append_kernel<float>, grid, dim3(256), 0, st, a);
}

}  // namespace cache
}  // namespace fibattn
