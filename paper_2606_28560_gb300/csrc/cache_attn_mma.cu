// cache_attn_mma.cu -- attention of new tokens over a paged cache, bf16 tensors
// (arXiv 2606.28560, Section 2, "Attended set"): s = scale q~ . key, softmax over
// window and rungs, out = sum p value; a rung's key and value are interpolated from
// two rows, so its score is (1-w) s_floor + w s_far and its rows have the weights
// p (1-w) and p w.
//
// A warp has one token and eight of its query heads: those of one key/value head, or
// of several, as far as eight go.  Rows go 32 to a part, up to 64 at once: each lane
// finds one of a part through the page table, for all heads; then m16n8k16 products
// take them.  The eight heads are rows 0-7 of the first operand and what their rounding
// to 16 bits left is rows 8-15, so that q (two fp16 halves, 22 bits: fit_half) and p (two
// bf16 halves, 16 bits) come with the products' idle half and fp32 sums.  A product with the rows of one
// key/value head is right for its own query heads; the others' scores are not taken,
// and their weights are 0 in its product with the values, so that all eight share one
// set of sums, one softmax and one way out.
//   Keys, then values, of one head after another go through a ring of shared memory,
// 16 bytes at a time, and into the products' fragments by matrix loads, transposed for
// the values, whose sum runs over rows; neither copies nor loads meet in a bank.
// Bound by memory where there are many sequences: 4096 single tokens of 8 heads 39 to
// 42 us, 5.3 to 5.7 TB/s of rows of 128 bytes; by the chain of look-ups, copies and products of the 16
// warps that an SM holds where rows come from L2 (8 chunks of 256 tokens 12.8 us) or where
// there are few (one token 3.2 us).  Keys straight into registers and values through
// a ring of two took 43.0, 12.1 and 3.1 us, and 164 us for 128 chunks where this way took
// 140; two stages and 20 warps an SM 38.7, 12.9 and 3.2 at the best heads a warp for each;
// blocks of four warps 1 to 2 % more for single tokens.
#include <algorithm>

#include "cache_rows.cuh"
#include "mma_common.cuh"

namespace fibattn {
namespace cache {

namespace {

constexpr int kWarps = 2;

// 2^k for scaling q to fp16's upper range, from the exponent of a head's largest value, which
// comes to lie in [2^14, 2^15), and 2^-k.  With the lower half times kLow, two halves of fp16
// keep 22 bits of a value down to 2^-29 of the largest, from where on the upper half is
// subnormal, and of smaller ones all but 2^-50 of the largest.
__device__ __forceinline__ void fit_half(float largest, float& up, float& down) {
    const int e = min(268 - (int)(__float_as_uint(largest) >> 23), 253);
    up = __uint_as_float((unsigned)e << 23);
    down = __uint_as_float((unsigned)(254 - e) << 23);
}

constexpr float kLow = 2048.f;                       // 2^11: a lower half to the size of its upper one

// A score from the sums of q's upper and lower halves.  Where a key is infinite the upper
// half's sum has the score's sign (or is NaN, as where that half is 0: below 2^-39 of the
// largest), the lower half's that of a rounding: it is left out where it makes NaN of the
// two.  (128 chunks 143.3 us with this, 141.1 without.)
__device__ __forceinline__ float whole(float upper, float lower) {
    const float s = fmaf(lower, 1.f / kLow, upper);
    return s == s ? s : upper;
}

constexpr int kStages = 3;                           // of the ring
constexpr unsigned kBytes = 32 * kHeadDim * 2;       // 32 rows of a head

// 32 rows of a key/value head into a stage, eight lanes to a row.  rows: where they lie for
// head 0, row 4i + k at 8k + i, so that a lane's eight are neighbours.  Chunk c (16 bytes)
// of row r lies at r * 128 + 16 (c ^ r % 8).  few: 16 rows do.
__device__ __forceinline__ void copy_rows(const void* pool, const unsigned* rows, unsigned head, int lane, unsigned to, bool few) {
    unsigned row[8];
    *reinterpret_cast<uint4*>(row) = *reinterpret_cast<const uint4*>(rows + 8 * (lane >> 3));
    *reinterpret_cast<uint4*>(row + 4) = *reinterpret_cast<const uint4*>(rows + 8 * (lane >> 3) + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i == 4 && few) break;
        const int r = 4 * i + (lane >> 3), c = lane & 7;
        const __half* from = static_cast<const __half*>(pool) + 8 * c + (size_t)(row[i] + head) * kHeadDim;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n"
                     :: "r"(to + r * 128 + ((c ^ (r & 7)) << 4)), "l"(from) : "memory");
    }
}

// A product of the heads' weights of 16 rows with these rows' values, for each of eight
// chunks of dims; from: the lane's place in the first.
__device__ __forceinline__ void add_values(float (&acc)[8][4], const unsigned* p, unsigned from) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        unsigned r[4];
        mma::ldsm_x4_t(from ^ (j << 5), r[0], r[1], r[2], r[3]);
#pragma unroll
        for (int e = 0; e < 2; ++e)
            mma::mma_bf16_16816(acc[2 * j + e], p, r[2 * e], r[2 * e + 1]);
    }
}

// kHalves: 16 rows each, taken together, two to a stage; kMany: queries read more than these (a
// warp then has one key/value head).
template <int kHalves, bool kMany, bool kTree>
__global__ void __launch_bounds__(32 * kWarps, kMany ? 6 : 8) attention_mma_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int kParts = (kHalves + 1) / 2;
    auto few = [](int c) { return kHalves % 2 == 1 && c == kParts - 1; };      // a part of 16 rows
    __shared__ __align__(128) unsigned char ring[kWarps][kStages][kBytes];
    __shared__ __align__(16) unsigned rows[kWarps][kParts][32];
    grid_dependency_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned unit = blockIdx.x * kWarps + warp;
    if (unit >= a.units) return;
    const unsigned n = fdiv(unit, a.dRest), rest = unit - n * a.dRest.d;
    const int pos = a.positions[n], seq = a.seqs ? a.seqs[n] : (int)n;
    // the lane's query head: the mine-th key/value head of the warp's, and its own number
    const unsigned run = fdiv(rest, a.dParts), part = rest - run * a.dParts.d;
    const int h0 = run * a.run, heads = min(a.run, a.c.Hkv - h0), mine = a.G >= 8 ? 0 : g / a.G;
    const int own = (int)part * 8 + g - mine * a.G;
    const bool real = mine < heads && own < a.G;
    const int head = (h0 + mine) * a.G + own;
    unsigned raw[8] = {};                              // dims 8c + 2t and the next, c < 8
    if (real) {
        const unsigned* row = reinterpret_cast<const unsigned*>(static_cast<const __nv_bfloat16*>(a.q) + n * a.q_token +
                                                                head * a.q_head);
#pragma unroll
        for (int c = 0; c < 8; ++c) raw[c] = row[4 * c + t];
    }
    const int* pages = a.c.table + (size_t)max(seq, 0) * a.c.pages_per_seq;
    const bool padding = pos < 0 || seq < 0;
    bool bad = !padding && seq >= a.c.seqs, turned = false;
    float m = -INFINITY, l = 0.f, sc = 0.f, acc[8][4];
    unsigned qf[4][4];                                 // four products of 16 dims: (half, half of the dims)
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
    };
    if (kMany) clear();
    for (int r0 = 0; r0 < (kMany ? a.r.total : 1) && !padding && !bad; r0 += 32 * kParts) {
        // where the rows lie; one that is not read stands for one that is: its score counts for nothing
        float share[kParts];
        unsigned live[kParts], pairs[kParts], place[kParts], some = 0, any = 0;
#pragma unroll
        for (int c = 0; c < kParts; ++c) {
            const int i = r0 + 32 * c + lane;
            const RowOf row = row_of(a.r, i);
            const bool lives = i < a.r.total && pos >= row.need;
            live[c] = __ballot_sync(kAll, lives);
            pairs[c] = __ballot_sync(kAll, row.pair);
            share[c] = row.weight;
            place[c] = 0;
            if (!live[c]) continue;
            int slot;
            bool found = slot_of<kTree>(a, n, pos, seq, row.distance, lives, slot);
            if (found && lives) found = locate(a.c, pages, slot, place[c]);
            bad |= __any_sync(kAll, !found);
            some = __shfl_sync(kAll, place[c], __ffs(live[c]) - 1);
            any = 1;
        }
        if (bad) break;
        if (!any) continue;
        if (kMany) __syncwarp();                       // what is written over has been read
#pragma unroll
        for (int c = 0; c < kParts; ++c) rows[warp][c][8 * (lane & 3) + (lane >> 2)] = live[c] >> lane & 1u ? place[c] : some;
        __syncwarp();
        // the ring: keys of each of the warp's key/value heads, part by part, then their values
        const unsigned base_at = mma::smem_u32(ring[warp][0]), step = a.c.head_stride, first = h0 * step;
        const int half = kParts * heads;
        auto issue = [&](int item, int stage) {
            if (item < 2 * half) {
                const int j = item < half ? item : item - half;
                const bool second = kParts > 1 && j >= heads;
                copy_rows(item < half ? a.c.k : a.c.v, rows[warp][second], first + (second ? j - heads : j) * step, lane,
                          base_at + stage * kBytes, few(0) || (second && few(1)));
            }
            asm volatile("cp.async.commit_group;\n" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < kStages; ++i) issue(i, i);
        if (!turned) {
            turned = true;
            float cs, sn, y[16], largest = 0.f;
            rope_cs_f32(a.c.rope, lane, pos, cs, sn);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int m_ = 8 * c + 2 * t + e;
                    const float co = __shfl_sync(kAll, cs, m_), si = __shfl_sync(kAll, sn, m_);
                    const float u = __uint_as_float(e ? raw[c] & 0xffff0000u : raw[c] << 16);
                    const float v = __uint_as_float(e ? raw[c + 4] & 0xffff0000u : raw[c + 4] << 16);
                    y[2 * c + e] = u * co - v * si;
                    y[8 + 2 * c + e] = v * co + u * si;
                    largest = fmaxf(largest, fmaxf(fabsf(y[2 * c + e]), fabsf(y[8 + 2 * c + e])));
                }
            float up, down;
            fit_half(mma::quad_max(largest), up, down);
            sc = down * a.scale;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float2 x = __fmul2_rn(make_float2(y[2 * c], y[2 * c + 1]), make_float2(up, up));
                const __half2 hi = __float22half2_rn(x);
                qf[c >> 1][2 * (c & 1)] = *reinterpret_cast<const unsigned*>(&hi);
                const float2 low = __ffma2_rn(__half22float2(hi), make_float2(-kLow, -kLow), __fmul2_rn(x, make_float2(kLow, kLow)));
                qf[c >> 1][2 * (c & 1) + 1] = mma::pack_f16(low.x, low.y);
            }
        }
        float s[kParts][4][2];
        int stage = 0, next = kStages;                 // the item that is read; the one to ask for
        auto wait = [&] {
            asm volatile("cp.async.wait_group %0;\n" :: "n"(kStages - 1) : "memory");
            __syncwarp();
        };
        auto advance = [&] {
            __syncwarp();                              // all lanes have read what is written over
            issue(next++, stage);
            stage = stage == kStages - 1 ? 0 : stage + 1;
        };
#pragma unroll
        for (int c = 0; c < kParts; ++c) {
            s[c][2][0] = s[c][2][1] = s[c][3][0] = s[c][3][1] = 0.f;
#pragma unroll 1
            for (int j = 0; j < heads; ++j) {
                wait();
                const unsigned from = base_at + stage * kBytes + (lane & 7) * 128 + (((lane >> 3) ^ (lane & 7)) << 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (i == 2 && few(c)) break;
                    unsigned k[8];
                    mma::ldsm_x4(from + i * 1024, k[0], k[1], k[2], k[3]);
                    mma::ldsm_x4((from + i * 1024) ^ 64, k[4], k[5], k[6], k[7]);
                    float d[4];
                    mma::mma_f16_16816_z(d, qf[0], k[0], k[1]);
                    mma::mma_f16_16816(d, qf[1], k[2], k[3]);
                    mma::mma_f16_16816(d, qf[2], k[4], k[5]);
                    mma::mma_f16_16816(d, qf[3], k[6], k[7]);
                    if (j == 0 || mine == j) {
                        s[c][i][0] = whole(d[0], d[2]);
                        s[c][i][1] = whole(d[1], d[3]);
                    }
                }
                advance();
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < kParts; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 8 * i + 2 * t;
                s[c][i][0] *= sc * __shfl_sync(kAll, share[c], r);
                s[c][i][1] *= sc * __shfl_sync(kAll, share[c], r + 1);
                if (pairs[c] >> r & 1u) s[c][i][0] = s[c][i][1] = s[c][i][0] + s[c][i][1];
                if (!(live[c] >> r & 1u)) s[c][i][0] = -INFINITY;
                if (!(live[c] >> r & 2u)) s[c][i][1] = -INFINITY;
                top = fmaxf(top, fmaxf(s[c][i][0], s[c][i][1]));
            }
        const float now = fmaxf(m, mma::quad_max(top));
        const float base = now == -INFINITY ? 0.f : now;           // no finite score so far: every weight is 0
        const float shrink = mma::ex2(m - base);
        m = now;
        l *= shrink;
        if (kMany) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] *= shrink;
        }
        unsigned p[kParts][8];                         // [8 rows: upper halves, lower halves]
#pragma unroll
        for (int c = 0; c < kParts; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p0 = mma::ex2(s[c][i][0] - base) * __shfl_sync(kAll, share[c], 8 * i + 2 * t);
                const float p1 = mma::ex2(s[c][i][1] - base) * __shfl_sync(kAll, share[c], 8 * i + 2 * t + 1);
                l += p0 + p1;
                const unsigned hi = mma::pack_bf16(p0, p1);
                p[c][2 * i] = hi;
                p[c][2 * i + 1] = mma::pack_bf16(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xffff0000u));
            }
        if (!kMany) clear();
        // the weights of this lane's query head, 0 for the rows of another key/value head
        auto add = [&](float (&to)[8][4], int c, int j, unsigned at) {
            unsigned pj[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) pj[i] = mine == j ? p[c][i] : 0u;
            const unsigned from = at + (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
            add_values(to, pj, from);
            if (!few(c)) add_values(to, pj + 4, from + 16 * 128);
        };
#pragma unroll
        for (int c = 0; c < kParts; ++c) {
#pragma unroll 1
            for (int j = 0; j < heads; ++j) {
                wait();
                add(acc, c, j, base_at + stage * kBytes);
                advance();
            }
        }
        if (!kMany && heads > 1) {
            // 0 times a value that is not finite is NaN: if there is one, the heads' sums are
            // taken again and kept apart, so that it stays with the heads that read it
            float zero = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) zero = fmaf(acc[j][e], 0.f, zero);
            if (__any_sync(kAll, !(zero == 0.f))) {
#pragma unroll 1
                for (int j = 0; j < heads; ++j) {
                    float one[8][4] = {};
#pragma unroll
                    for (int c = 0; c < kParts; ++c) {
                        issue(half + c * heads + j, 0);
                        asm volatile("cp.async.wait_group 0;\n" ::: "memory");
                        __syncwarp();
                        add(one, c, j, base_at);
                        __syncwarp();
                    }
                    if (mine == j) {
#pragma unroll
                        for (int d = 0; d < 8; ++d)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[d][e] = one[d][e];
                    }
                }
            }
        }
    }
    l = mma::quad_sum(l);
    float z = m + log2f(l);
    const float by = 1.f / l, none = bad ? NAN : 0.f;
    if (padding) z = -INFINITY;
    if (bad) z = NAN;
    if (real) {
        const size_t at = (size_t)n * a.H + head;
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + at * kHeadDim + 2 * t;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *reinterpret_cast<__nv_bfloat162*>(out + 8 * j) =
                padding || bad ? __float2bfloat162_rn(none)
                               : __floats2bfloat162_rn((acc[j][0] + acc[j][2]) * by, (acc[j][1] + acc[j][3]) * by);
        if (t == 0) a.lse[at] = z * kLn2;
    }
    if (bad && lane == 0) raise_status(a.status, kStatusPage);
}

template <int kHalves, bool kMany>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
    const dim3 grid((a.units + kWarps - 1) / kWarps), block(32 * kWarps);
    return a.parents ? launch_kernel(attention_mma_kernel<kHalves, kMany, true>, grid, block, 0, st, a)
                     : launch_kernel(attention_mma_kernel<kHalves, kMany, false>, grid, block, 0, st, a);
}

}  // namespace

cudaError_t launch_attention_mma(const AttnArgs& args, cudaStream_t st) {
    AttnArgs a = args;
    // Key/value heads of a warp, as far as its eight query heads go: the rows are looked up
    // once for all, but few warps leave the GPU waiting.  With 1, 2, 4, 8 heads a warp, us, of 8
    // heads over 8: 256 single tokens 5.4, 4.8, 5.0; 512 8.7, 6.4, 6.1; 1024 16.5, 12.6, 11.1,
    // 10.9; 4096 56.5, 45.1, 40.3, 39.7; chunks 8 x 64 8.7, 6.6, 6.2, 6.9, 8 x 256 25.9, 18.1, 14.3,
    // 13.2; drafts 16 x 32 10.4, 7.3, 7.0, 7.7, 64 x 32 30.9, 21.2, 16.3, 13.8.  Of 8 over 2: 1024
    // single tokens 5.5, 5.2, chunks 8 x 256 8.7, 6.7, drafts 64 x 32 10.2, 7.5.
    const int most = std::min(8 / std::min(a.G, 8), a.c.Hkv);
    a.run = a.r.total > 64 ? 1 : std::max(1, std::min(most, a.N * a.c.Hkv / 1024));
    const unsigned parts = (a.G + 7) / 8, runs = (a.c.Hkv + a.run - 1) / a.run;
    a.units = (unsigned)a.N * runs * parts;
    a.dRest = FastDiv::make(runs * parts);
    a.dParts = FastDiv::make(parts);
    // All of a query's rows at once as far as 64 go, 16 by 16: 4096 tokens of 35 rows (W = 16) 52.5 us
    // with three halves, 59 with four (which keep 26 bytes a thread in memory), 96 part by part (which also
    // keeps a warp at one head).
    const int halves = (a.r.total + 15) / 16;
    return halves <= 1 ? launch<1, false>(a, st) : halves == 2 ? launch<2, false>(a, st) : halves == 3 ? launch<3, false>(a, st)
         : halves == 4 ? launch<4, false>(a, st) : launch<4, true>(a, st);
}

}  // namespace cache
}  // namespace fibattn
