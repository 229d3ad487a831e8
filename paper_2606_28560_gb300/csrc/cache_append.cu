// cache_append.cu -- keys and values of new tokens into a paged cache, the keys
// rotated on the way: k~ = R(pos) k (arXiv 2606.28560, Section 2: RoPE at true
// positions, before the gather), values as they are.
//
// Bound by memory: each value is read and written once.  A warp has eight rows (heads
// of one token, or of several), four lanes to a row, so that a rotation's pair stays
// in its lane.  What is read does not wait for where it goes: the loads are under way
// while the warp looks up pages and evaluates its tokens' 32 angles, one to a lane,
// once for all heads.  64 prompts of 1024 tokens (8 heads, bf16, 269 MB) take 42.0 us,
// 6.4 TB/s; a token's thread with all its heads took 46.8, two and four steps of a warp
// at once 2 and 18 % longer, blocks of eight warps 2 % less there but a batch of 256
// single tokens 3.0 us instead of 2.5.
#include "cache.cuh"

namespace fibattn {
namespace cache {

namespace {

constexpr int kWarps = 4;
constexpr unsigned kAll = 0xffffffffu;

// A lane's 16 of a row's 64 elements, 8c .. 8c+7 and 32 more, as they lie in memory.
template <typename T> struct Part { uint4 x[sizeof(T)]; };
template <typename T>
__device__ __forceinline__ void load_part(const T* row, int c, Part<T>& p) {
    constexpr int n = (int)sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        p.x[i] = reinterpret_cast<const uint4*>(row + 8 * c)[i];
        p.x[n + i] = reinterpret_cast<const uint4*>(row + kHalf + 8 * c)[i];
    }
}
template <typename T>
__device__ __forceinline__ void store_part(T* row, int c, const Part<T>& p) {
    constexpr int n = (int)sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        reinterpret_cast<uint4*>(row + 8 * c)[i] = p.x[i];
        reinterpret_cast<uint4*>(row + kHalf + 8 * c)[i] = p.x[n + i];
    }
}
__device__ __forceinline__ void unpack(const Part<float>& p, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(x + 4 * i) = p.x[i];
}
__device__ __forceinline__ void unpack(const Part<__nv_bfloat16>& p, float* x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned w[4] = {p.x[i].x, p.x[i].y, p.x[i].z, p.x[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
            x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(32 * kWarps) append_kernel(const __grid_constant__ AppendArgs a) {
    using R = typename RotOf<T>::type;
    __shared__ __align__(16) float turn[kWarps][8][2][kHalf];      // cos and sin of the tokens' angles
    grid_dependency_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, s = lane >> 2, c = lane & 3;
    const int token = a.per > 1 ? s / a.c.Hkv : 0, h0 = s - token * a.c.Hkv;
    const long long first = ((long long)blockIdx.x * kWarps + warp) * a.per, n = first + token;
    if (first >= a.N) return;
    bool there = token < a.per && n < a.N && h0 < a.c.Hkv;
    const T* from_k = static_cast<const T*>(a.k) + n * a.k_token;
    const T* from_v = static_cast<const T*>(a.v) + n * a.v_token;
    Part<T> k, v;
    int pos = -1;
    unsigned row = 0;
    if (there) {
        load_part(from_k + h0 * a.k_head, c, k);
        load_part(from_v + h0 * a.v_head, c, v);
        pos = a.positions[n];
        const int seq = a.seqs ? a.seqs[n] : (int)n, slot = a.slots ? a.slots[n] : pos;
        if (pos < 0 || seq < 0) {
            there = false;                             // padding
        } else if (seq >= a.c.seqs || !locate(a.c, a.c.table + (size_t)seq * a.c.pages_per_seq, slot, row)) {
            there = false;
            if (c == 0 && h0 == 0) raise_status(a.status, kStatusPage);
        }
    }
    for (int j = 0; j < a.per; ++j) {                  // the first head of token j is in lane 4 j Hkv
        const int at = __shfl_sync(kAll, pos, a.per > 1 ? 4 * j * a.c.Hkv : 0);
        rope_cs_f32(a.c.rope, lane, max(at, 0), turn[warp][j][0][lane], turn[warp][j][1][lane]);
    }
    __syncwarp();
    if (!there) return;
    const float *cs = turn[warp][token][0] + 8 * c, *sn = turn[warp][token][1] + 8 * c;
    float largest = 0.f;
    for (int h = h0; h < a.c.Hkv; h += 8) {            // (more than once for a token of more than eight heads)
        if (h != h0) {
            load_part(from_k + h * a.k_head, c, k);
            load_part(from_v + h * a.v_head, c, v);
        }
        const size_t to = (size_t)(row + h * a.c.head_stride) * kHeadDim;
        float x[16];
        unpack(k, x);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float p = x[u], q = x[8 + u];
            x[u] = p * cs[u] - q * sn[u];
            x[8 + u] = q * cs[u] + p * sn[u];
            largest = fmaxf(largest, fmaxf(fabsf(x[u]), fabsf(x[8 + u])));
        }
        store_chunk(static_cast<R*>(a.c.k) + to, c, x);
        store_part(static_cast<T*>(a.c.v) + to, c, v);
    }
    if (sizeof(R) == 2 && largest >= 65520.f) raise_status(a.status, kStatusRange);   // rounds to infinity in fp16
}

}  // namespace

cudaError_t launch_append(const AppendArgs& args, bool bf16, cudaStream_t st) {
    AppendArgs a = args;
    a.per = a.c.Hkv > 4 ? 1 : 8 / a.c.Hkv;
    const long long warps = ((long long)a.N + a.per - 1) / a.per;
    const dim3 grid((unsigned)((warps + kWarps - 1) / kWarps)), block(32 * kWarps);
    return bf16 ? launch_kernel(append_kernel<__nv_bfloat16>, grid, block, 0, st, a)
                : launch_kernel(append_kernel<float>, grid, block, 0, st, a);
}

}  // namespace cache
}  // namespace fibattn
