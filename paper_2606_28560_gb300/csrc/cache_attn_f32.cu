// cache_attn_f32.cu -- attention of new tokens over a paged cache, fp32 (arXiv
// 2606.28560, Section 2, "Attended set"): s = scale q~ . key, softmax over window and
// rungs, out = sum p value; a rung's key and value are interpolated from two rows, so
// its score is (1-w) s_floor + w s_far and its rows have weights p (1-w) and p w.
//
// A warp has one token and key/value head, its group of query heads or a part of it.
// Rows go 32 to a part: each lane finds one of a part through the page table; then all
// lanes load keys, eight lanes to a row (32 bytes of it each), while the values are
// copied to shared memory.  Eight partial dot products per lane are exchanged so that a
// lane ends with the score of the row it looked up, and the softmax is one value per
// lane and part.  The weights of all heads are kept, then the values are read.
// Bound by memory where there are many sequences: 2048 single tokens of 8 heads 38.1 us,
// 5.9 TB/s; by the chain of look-ups and loads where there are few: one token 3.3 us.
#include <algorithm>

#include "cache_rows.cuh"
#include "mma_common.cuh"

namespace fibattn {
namespace cache {

namespace {

constexpr int kHeads = 8;                            // query heads of a warp, at most
constexpr int warps_of(int parts) { return parts == 1 ? 4 : 2; }   // of a block: 45 and 41 KB of shared memory

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

__device__ __forceinline__ void load_keys(const float* from, float* x) {
    unsigned* u = reinterpret_cast<unsigned*>(x);
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
                 : "l"(from));
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

// The four groups' sums of a lane's eight dims (4c .. 4c+3 and 32 more) are added, each
// lane keeping two, and written, times `by`.
__device__ __forceinline__ void write_out(float* out, const float (&acc)[8], float by, int lane) {
    const bool up2 = lane & 16, up1 = lane & 8;
    float o[4], x[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float keep = up2 ? acc[j + 4] : acc[j], give = up2 ? acc[j] : acc[j + 4];
        o[j] = keep + __shfl_xor_sync(kAll, give, 16);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float keep = up1 ? o[j + 2] : o[j], give = up1 ? o[j] : o[j + 2];
        x[j] = keep + __shfl_xor_sync(kAll, give, 8);
    }
    *reinterpret_cast<float2*>(out + (up2 ? kHalf : 0) + 4 * (lane & 7) + (up1 ? 2 : 0)) = make_float2(x[0] * by, x[1] * by);
}

template <int kParts>
struct Shared {
    float values[kParts][32][kHeadDim];              // in the order of the lanes that found the rows
    float p[kParts][kHeads][32];                     // scores, then weights, in the same order
    float q[kHeads][kHeadDim];                       // rotated queries
};

// kParts: of 32 rows each, taken together; kMany: queries read more than these (a warp then
// has one query head).
template <int kParts, bool kMany, bool kTree>
__global__ void __launch_bounds__(32 * warps_of(kParts), kParts == 1 ? 4 : 5) attention_f32_kernel(const __grid_constant__ AttnArgs a) {
    __shared__ __align__(16) Shared<kParts> shared[warps_of(kParts)];
    grid_dependency_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 7, group = lane >> 3;
    const unsigned unit = blockIdx.x * warps_of(kParts) + warp;
    if (unit >= a.units) return;
    Shared<kParts>& sh = shared[warp];
    const unsigned n = fdiv(unit, a.dRest), rest = unit - n * a.dRest.d, h = fdiv(rest, a.dParts);
    const int part = rest - h * a.dParts.d, g0 = h * a.G + part * a.run, heads = kMany ? 1 : min(a.run, a.G - part * a.run);
    const int pos = a.positions[n], seq = a.seqs ? a.seqs[n] : (int)n;
    const float* q = static_cast<const float*>(a.q) + n * a.q_token + g0 * a.q_head;
    const float qx = q[lane], qy = q[lane + kHalf];
    float* out = static_cast<float*>(a.out) + ((size_t)n * a.H + g0) * kHeadDim;
    float* lse = a.lse + (size_t)n * a.H + g0;
    const int* pages = a.c.table + (size_t)max(seq, 0) * a.c.pages_per_seq;
    const bool padding = pos < 0 || seq < 0;
    bool bad = !padding && seq >= a.c.seqs, turned = false;
    float m = -INFINITY, l = 0.f, acc[8];            // (kMany: over the rows so far)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    for (int r0 = 0; r0 < (kMany ? a.r.total : 1) && !padding && !bad; r0 += 32 * kParts) {
        // where the rows lie; one that is not read stands for one that is: its score counts for nothing
        float share[kParts];
        bool live[kParts], pair[kParts], any = false;
        unsigned at[kParts], some = 0;
#pragma unroll
        for (int b = 0; b < kParts; ++b) {
            // lane (group, c) has row 4c + group: the scores are exchanged to that order
            const int i = r0 + 32 * b + 4 * c + group;
            const RowOf row = row_of(a.r, i);
            live[b] = i < a.r.total && pos >= row.need;
            pair[b] = row.pair;
            share[b] = row.weight;
            at[b] = 0;
            const unsigned alive = __ballot_sync(kAll, live[b]);
            if (!alive) continue;
            int slot;
            bool found = slot_of<kTree>(a, n, pos, seq, row.distance, live[b], slot);
            if (found && live[b]) found = locate(a.c, pages, slot, at[b]);
            bad |= __any_sync(kAll, !found);
            some = __shfl_sync(kAll, at[b], __ffs(alive) - 1);
            any = true;
        }
        if (bad) break;
        if (!any) continue;
        if (kMany) __syncwarp();                     // what is written over has been read
        // the second part has 16 rows or fewer: the first four of every eight in the lanes' order
        const bool few = kParts > 1 && a.r.total <= 48;
        float k[8][8];
#pragma unroll
        for (int b = 0; b < kParts; ++b) {
            at[b] = (live[b] ? at[b] : some) + h * a.c.head_stride;
            if (b == 0)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    load_keys(static_cast<const float*>(a.c.k) + (size_t)__shfl_sync(kAll, at[0], 8 * group + j) * kHeadDim + 8 * c, k[j]);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (b > 0 && j % 4 >= 2 && few) continue;
                const int r = 2 * j + (lane >> 4);
                const float* from = static_cast<const float*>(a.c.v) + (size_t)__shfl_sync(kAll, at[b], r) * kHeadDim + 4 * (lane & 15);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n"
                             :: "r"(mma::smem_u32(&sh.values[b][r][4 * (lane & 15)])), "l"(from) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
        if (!turned) {
            turned = true;
            float cs, sn;
            rope_cs_f32(a.c.rope, lane, pos, cs, sn);
            // (roundings as written, so that a head has the same bits wherever in a warp it is)
            auto turn = [&](float* to, float x, float y) {
                to[lane] = __fmul_rn(__fmaf_rn(x, cs, -__fmul_rn(y, sn)), a.scale);
                to[lane + kHalf] = __fmul_rn(__fmaf_rn(y, cs, __fmul_rn(x, sn)), a.scale);
            };
            turn(sh.q[0], qx, qy);
#pragma unroll 4
            for (int g = 1; g < heads; ++g) turn(sh.q[g], q[g * a.q_head + lane], q[g * a.q_head + lane + kHalf]);
            __syncwarp();
        }
#pragma unroll
        for (int b = 0; b < kParts; ++b) {
            if (b > 0)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < 4 || !few)
                        load_keys(static_cast<const float*>(a.c.k) + (size_t)__shfl_sync(kAll, at[b], 8 * group + j) * kHeadDim + 8 * c, k[j]);
            for (int g = 0; g < heads; ++g) {
                const float4 qa = *reinterpret_cast<const float4*>(&sh.q[g][8 * c]);
                const float4 qb = *reinterpret_cast<const float4*>(&sh.q[g][8 * c + 4]);
                float s[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float2 t = __fmul2_rn(make_float2(k[j][0], k[j][1]), make_float2(qa.x, qa.y));
                    t = __ffma2_rn(make_float2(k[j][2], k[j][3]), make_float2(qa.z, qa.w), t);
                    t = __ffma2_rn(make_float2(k[j][4], k[j][5]), make_float2(qb.x, qb.y), t);
                    t = __ffma2_rn(make_float2(k[j][6], k[j][7]), make_float2(qb.z, qb.w), t);
                    s[j] = t.x + t.y;
                }
                float score = sum_own(s, c) * share[b];
                const float other = __shfl_xor_sync(kAll, score, 8);
                if (pair[b]) score += other;
                sh.p[b][g][lane] = live[b] ? score : -INFINITY;
            }
        }
        for (int g = 0; g < heads; ++g) {            // (each lane reads what it wrote)
            float top = sh.p[0][g][lane];
            if (kParts > 1) top = fmaxf(top, sh.p[kParts - 1][g][lane]);
            const float now = fmaxf(kMany ? m : -INFINITY, warp_max(top));
            const float base = now == -INFINITY ? 0.f : now;       // no finite score so far: every weight is 0
            float p[kParts], sum = 0.f;
#pragma unroll
            for (int b = 0; b < kParts; ++b) sum += p[b] = exp2f(sh.p[b][g][lane] - base) * share[b];
            if (kMany) {
                const float shrink = exp2f(m - base);
                l = l * shrink + sum;
                m = now;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] *= shrink;
            } else {
                l = warp_sum(sum);
                if (lane == 0) lse[g] = (now + log2f(l)) * kLn2;
            }
#pragma unroll
            for (int b = 0; b < kParts; ++b) sh.p[b][g][lane] = kMany ? p[b] : p[b] / l;
        }
        asm volatile("cp.async.wait_group 0;\n" ::: "memory");
        __syncwarp();
        // rows 8 group + j: dims 4c .. 4c+3 and 32 more; one part's stay in registers for all heads
        float v[8][8];
        auto fetch = [&](int b, int j) {
            *reinterpret_cast<float4*>(v[j]) = *reinterpret_cast<const float4*>(&sh.values[b][8 * group + j][4 * c]);
            *reinterpret_cast<float4*>(v[j] + 4) = *reinterpret_cast<const float4*>(&sh.values[b][8 * group + j][kHalf + 4 * c]);
        };
        if (kParts == 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) fetch(0, j);
        }
        for (int g = 0; g < heads; ++g) {
            if (!kMany) {
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = 0.f;
            }
#pragma unroll
            for (int b = 0; b < kParts; ++b) {
                float p[8];
                *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(&sh.p[b][g][8 * group]);
                *reinterpret_cast<float4*>(p + 4) = *reinterpret_cast<const float4*>(&sh.p[b][g][8 * group + 4]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (b > 0 && j == 4 && few) break;
                    if (kParts > 1) fetch(b, j);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float2 t = __ffma2_rn(make_float2(p[j], p[j]), make_float2(v[j][e], v[j][e + 1]),
                                                    make_float2(acc[e], acc[e + 1]));
                        acc[e] = t.x;
                        acc[e + 1] = t.y;
                    }
                }
            }
            if (!kMany) write_out(out + g * kHeadDim, acc, 1.f, lane);
        }
    }
    if (padding || bad) {
        for (int g = 0; g < heads; ++g) {
            out[g * kHeadDim + lane] = out[g * kHeadDim + kHalf + lane] = bad ? NAN : 0.f;
            if (lane == 0) lse[g] = bad ? NAN : -INFINITY;
        }
        if (bad && lane == 0) raise_status(a.status, kStatusPage);
    } else if (kMany) {
        l = warp_sum(l);
        write_out(out, acc, 1.f / l, lane);
        if (lane == 0) lse[0] = (m + log2f(l)) * kLn2;
    }
}

template <int kParts, bool kMany>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
    constexpr int warps = warps_of(kParts);
    const dim3 grid((a.units + warps - 1) / warps), block(32 * warps);
    return a.parents ? launch_kernel(attention_f32_kernel<kParts, kMany, true>, grid, block, 0, st, a)
                     : launch_kernel(attention_f32_kernel<kParts, kMany, false>, grid, block, 0, st, a);
}

}  // namespace

cudaError_t launch_attention_f32(const AttnArgs& args, cudaStream_t st) {
    AttnArgs a = args;
    // Query heads of a warp: they share the rows' look-up and loads, but few warps leave the GPU
    // waiting.  One token each, us: 256 tokens of 8 heads over 1 with 1, 2, 4, 8 heads a warp 5.6,
    // 5.2, 5.9, 8.5.  With 1, 2, 4 heads of 8 over 2: 1024 tokens 13.9, 10.5, 9.0; 4096 52.6, 40.5, 40.0;
    // chunks 8 x 256 23.8, 18.2, 14.1; drafts 64 x 32 27.8, 20.1, 15.7.
    const int all = a.N * a.H;
    a.run = a.r.total > 64 || (a.r.total > 32 && a.G == 1) || all < 2048 ? 1 : std::min({a.G, kHeads, std::max(2, all / 2048)});
    const unsigned parts = (a.G + a.run - 1) / a.run;
    a.units = (unsigned)a.N * a.c.Hkv * parts;
    a.dRest = FastDiv::make(a.c.Hkv * parts);
    a.dParts = FastDiv::make(parts);
    // More than 32 rows part by part, but up to 64 at once where heads share them: 1024 tokens with
    // every rung (37 rows), us: 8 heads over 8 28.8 and 34.2, 8 over 2 22.3 and 18.1.  (Not by the heads
    // of a warp: a token would have other bits in another batch.)
    return a.r.total <= 32 ? launch<1, false>(a, st) : a.r.total <= 64 && a.G > 1 ? launch<2, false>(a, st) : launch<1, true>(a, st);
}

}  // namespace cache
}  // namespace fibattn
