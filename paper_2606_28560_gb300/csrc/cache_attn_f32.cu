// cache_attn_f32.cu -- attention of new tokens over a paged cache, fp32 (arXiv
// 2606.28560, Section 2, "Attended set"): s = scale q~ . key, softmax over window and rungs,
// out = sum p value; a rung's key and value are interpolated from two rows, so its
// score is (1-w) s_floor + w s_far and its rows have weights p (1-w) and p w.
//
// A warp has one token and key/value head (its group of query heads, or a part of
// it).  32 rows at a time: each lane finds one row through the page table; then all
// lanes load rows, eight lanes to a row (32 bytes of it each), four rows
// to an instruction, all of keys and values at once.  Eight partial dot products per
// lane are exchanged so that a lane ends with the score of the row it looked up, and
// the softmax is one value per lane.
#include <algorithm>

#include "cache_rows.cuh"

namespace fibattn {
namespace cache {

namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kAll, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}

// Eight elements of a row.
struct Raw { float4 lo, hi; };
__device__ __forceinline__ Raw load_raw(const void* pool, unsigned row, int c) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(pool) + (size_t)row * kHeadDim + 8 * c);
    return {p[0], p[1]};
}

// v[i] summed over the eight lanes of a group, each lane keeping i = its number:
// halves are exchanged, 7 shuffles instead of 24.
__device__ __forceinline__ float sum_own(float (&v)[8], int c) {
#pragma unroll
    for (int half = 4; half > 0; half >>= 1) {
        const bool upper = c & half;
#pragma unroll
        for (int j = 0; j < half; ++j) {
            const float keep = upper ? v[j + half] : v[j], give = upper ? v[j] : v[j + half];
            v[j] = keep + __shfl_xor_sync(kAll, give, half);
        }
    }
    return v[0];
}

// Running softmax of one query head over the rows so far: m the largest score, l the
// sum of weights (each lane its own rows'), acc the values (each lane's rows and dims).
struct Running { float m, l, acc[8]; };

// One group of up to 32 rows, loaded: scores, weights, values for one query head.
__device__ __forceinline__ void attend(const Raw (&k)[8], const Raw (&v)[8], const float* q, int c, bool live,
                                       const RowOf& row, Running& run) {
    float s[8];
    float qc[8];
    *reinterpret_cast<float4*>(qc) = *reinterpret_cast<const float4*>(q + 8 * c);
    *reinterpret_cast<float4*>(qc + 4) = *reinterpret_cast<const float4*>(q + 8 * c + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x[8] = {k[i].lo.x, k[i].lo.y, k[i].lo.z, k[i].lo.w, k[i].hi.x, k[i].hi.y, k[i].hi.z, k[i].hi.w};
        float2 t = __fmul2_rn(make_float2(x[0], x[1]), make_float2(qc[0], qc[1]));
#pragma unroll
        for (int j = 1; j < 4; ++j)
            t = __ffma2_rn(make_float2(x[2 * j], x[2 * j + 1]), make_float2(qc[2 * j], qc[2 * j + 1]), t);
        s[i] = t.x + t.y;
    }
    float score = sum_own(s, c) * row.weight;
    const float other = __shfl_xor_sync(kAll, score, 8);
    if (row.pair) score += other;
    if (!live) score = -INFINITY;
    const float m = fmaxf(run.m, warp_max(score));
    const float base = m == -INFINITY ? 0.f : m;      // no finite score so far: every weight is 0
    const float p = live ? exp2f(score - base) * row.weight : 0.f;
    const float shrink = exp2f(run.m - base);
    run.l = run.l * shrink + p;
    run.m = m;
    const int group = threadIdx.x & 24;
#pragma unroll
    for (int j = 0; j < 8; ++j) run.acc[j] *= shrink;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float w = __shfl_sync(kAll, p, group + i);
        const float x[8] = {v[i].lo.x, v[i].lo.y, v[i].lo.z, v[i].lo.w, v[i].hi.x, v[i].hi.y, v[i].hi.z, v[i].hi.w};
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float2 t = __ffma2_rn(make_float2(w, w), make_float2(x[j], x[j + 1]),
                                        make_float2(run.acc[j], run.acc[j + 1]));
            run.acc[j] = t.x;
            run.acc[j + 1] = t.y;
        }
    }
}

template <bool kTree>
__global__ void __launch_bounds__(32 * kWarps) attention_kernel(const __grid_constant__ AttnArgs a) {
    __shared__ __align__(16) float qs[kWarps][kHeadDim];
    grid_dependency_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 7, group = lane >> 3;
    const long long unit = blockIdx.x * (long long)kWarps + warp;
    if (unit >= (long long)a.N * a.c.Hkv * a.parts) return;
    const int part = (int)(unit % a.parts), h = (int)(unit / a.parts % a.c.Hkv), n = (int)(unit / a.parts / a.c.Hkv);
    const int g0 = h * a.G + part * a.per_part, g1 = h * a.G + min(a.G, (part + 1) * a.per_part);
    float* out = static_cast<float*>(a.out) + (size_t)n * a.H * kHeadDim;
    float* lse = a.lse + (size_t)n * a.H;
    const int pos = a.positions[n], seq = a.seqs ? a.seqs[n] : n;
    const int* pages = a.c.table + (size_t)max(seq, 0) * a.c.pages_per_seq;
    bool bad = seq >= a.c.seqs;
    const bool padding = pos < 0 || seq < 0;
    float cs, sn;
    rope_cs_f32(a.c.rope, lane, max(pos, 0), cs, sn);
    for (int g = g0; g < g1; ++g) {
        Running run;
        run.m = -INFINITY;
        run.l = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) run.acc[j] = 0.f;
        if (!padding && !bad) {
            const float* q = static_cast<const float*>(a.q) + n * a.q_token + g * a.q_head;
            const float x = q[lane] * a.scale, y = q[lane + kHalf] * a.scale;
            __syncwarp();
            qs[warp][lane] = x * cs - y * sn;
            qs[warp][lane + kHalf] = y * cs + x * sn;
            __syncwarp();
        }
        for (int r0 = 0; r0 < a.r.total && !padding && !bad; r0 += 32) {
            // lane (group, c) has row 4c + group: the scores are exchanged to that order
            const int i = r0 + 4 * c + group;
            const RowOf row = row_of(a.r, i);
            const bool live = i < a.r.total && pos >= row.need;
            if (!__any_sync(kAll, live)) continue;
            int slot;
            unsigned at = 0;
            bool found = slot_of<kTree>(a, n, pos, row.distance, live, slot);
            if (found && live) found = locate(a.c, pages, slot, at);
            bad = __any_sync(kAll, !found);
            if (bad) break;
            at += h * a.c.head_stride;
            Raw k[8], v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned from = __shfl_sync(kAll, at, 8 * group + j);
                const bool there = __shfl_sync(kAll, (int)live, 8 * group + j);
                k[j] = v[j] = Raw{};
                if (there) {
                    k[j] = load_raw(a.c.k, from, c);
                    v[j] = load_raw(a.c.v, from, c);
                }
            }
            attend(k, v, qs[warp], c, live, row, run);
        }
        // the four groups' values are added, each lane keeping two dims
        const bool up2 = group & 2, up1 = group & 1;
        float o[4], o2[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float keep = up2 ? run.acc[j + 4] : run.acc[j], give = up2 ? run.acc[j] : run.acc[j + 4];
            o[j] = keep + __shfl_xor_sync(kAll, give, 16);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float keep = up1 ? o[j + 2] : o[j], give = up1 ? o[j] : o[j + 2];
            o2[j] = keep + __shfl_xor_sync(kAll, give, 8);
        }
        float l = warp_sum(run.l), z = run.m + log2f(l);
        float by = 1.f / l;
        if (padding) { by = 0.f; z = -INFINITY; }
        if (bad && !padding) by = z = NAN;
        const int d = 8 * c + 4 * up2 + 2 * up1;
        *reinterpret_cast<float2*>(out + (size_t)g * kHeadDim + d) = make_float2(o2[0] * by, o2[1] * by);
        if (lane == 0) lse[g] = z * kLn2;
    }
    if (bad && !padding && lane == 0) raise_status(a.status, kStatusPage);
}

}  // namespace

cudaError_t launch_attention_f32(const AttnArgs& args, cudaStream_t st) {
    AttnArgs a = args;
    const long long units = (long long)a.N * a.c.Hkv;
    a.parts = (int)std::max(1LL, std::min<long long>(a.G, 152LL * 16 / units));
    a.per_part = (a.G + a.parts - 1) / a.parts;
    a.parts = (a.G + a.per_part - 1) / a.per_part;
    const dim3 grid((unsigned)((units * a.parts + kWarps - 1) / kWarps)), block(32 * kWarps);
    return a.parents ? launch_kernel(attention_kernel<true>, grid, block, 0, st, a)
                     : launch_kernel(attention_kernel<false>, grid, block, 0, st, a);
}

}  // namespace cache
}  // namespace fibattn
