// cache_attn_mma.cu -- attention of new tokens over a paged cache, bf16 tensors
// (arXiv 2606.28560, Section 2, "Attended set"): s = scale q~ . key, softmax over
// window and rungs, out = sum p value; a rung's key and value are interpolated from
// two rows, so its score is (1-w) s_floor + w s_far and its rows have the weights
// p (1-w) and p w.
//
// A warp has one token and eight of its query heads: those of one key/value head, or
// of several (kRun), as far as eight go.  32 rows at a time: each lane finds one row
// through the page table, for all heads; then the rows are loaded straight into the
// fragments of m16n8k16 products, one key/value head ahead of the products.  The
// eight heads are rows 0-7 of the first operand and what their rounding to 16 bits
// left is rows 8-15, so that q (two fp16 halves, 22 bits) and p (two bf16 halves, 16
// bits) come with the products' idle half and fp32 sums.  A product with the rows of
// one key/value head is right for its own query heads; the others' scores are not
// taken, and their weights are 0 in its product with the values, so that all eight
// share one set of sums, one softmax and one way out.
//   Scores: a lane of column n holds 16 of row n's 64 dims, as they lie in memory;
// the order of dims within a product is free as long as q has the same.
//   Values: a lane's four rows of a 16-row product are those whose weights it holds
// after the scores; it loads the same eight dims of each and pairs them by byte
// permutes; product j takes dim j of the eight, so a lane ends with 16 dims in order.
#include <algorithm>

#include "cache_rows.cuh"
#include "mma_common.cuh"

namespace fibattn {
namespace cache {

namespace {

constexpr int kWarps = 4;

// 2^k for scaling q to fp16's upper range, from the exponent of its largest value,
// and 2^-k: halves of fp16 then keep 22 bits of every q, whatever its size.
__device__ __forceinline__ void fit_half(float largest, float& up, float& down) {
    const int e = min(268 - (int)(__float_as_uint(largest) >> 23), 253);
    up = __uint_as_float((unsigned)e << 23);
    down = __uint_as_float((unsigned)(254 - e) << 23);
}

struct Part { uint4 x[8]; };                         // a lane's part of 32 rows' keys or values
struct Places { unsigned k[4], v[8]; };              // where they lie, for key/value head 0

__device__ __forceinline__ void load_keys(const AttnArgs& a, const Places& p, unsigned head, int t, Part& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4* row = reinterpret_cast<const uint4*>(
            static_cast<const __half*>(a.c.k) + 8 * t + (size_t)(p.k[i] + head) * kHeadDim);
        b.x[2 * i] = row[0];
        b.x[2 * i + 1] = row[4];
    }
}
__device__ __forceinline__ int value_row(int i, int t) { return 8 * (i >> 1) + 2 * t + (i & 1); }
__device__ __forceinline__ void load_values(const AttnArgs& a, const Places& p, unsigned head, int g, Part& b) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        b.x[i] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.c.v) + 8 * g +
                                                 (size_t)(p.v[i] + head) * kHeadDim);
}

// A product of the heads' weights of 16 rows with these rows' values, for each of eight
// dims; kFirst: not added to anything.
template <bool kFirst>
__device__ __forceinline__ void add_values(float (&acc)[8][4], const unsigned* p, const uint4* v) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        unsigned r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = w == 0 ? v[i].x : w == 1 ? v[i].y : w == 2 ? v[i].z : v[i].w;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const unsigned pick = e ? 0x7632 : 0x5410, b0 = __byte_perm(r[0], r[1], pick), b1 = __byte_perm(r[2], r[3], pick);
            if (kFirst) mma::mma_bf16_16816_z(acc[2 * w + e], p, b0, b1);
            else mma::mma_bf16_16816(acc[2 * w + e], p, b0, b1);
        }
    }
}

// kRun: key/value heads of a warp; kMany: queries read more than 32 rows.
template <int kRun, bool kMany, bool kTree>
__global__ void __launch_bounds__(32 * kWarps, 4) attention_mma_kernel(const __grid_constant__ AttnArgs a) {
    __shared__ __align__(16) float turn[kWarps][2][kHalf];         // cos and sin of the token's angles
    grid_dependency_sync();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned unit = blockIdx.x * kWarps + warp;
    if (unit >= a.units) return;
    const unsigned n = fdiv(unit, a.dRest), rest = unit - n * a.dRest.d;
    const int pos = a.positions[n], seq = a.seqs ? a.seqs[n] : (int)n;
    // the lane's query head: the mine-th key/value head of the warp's, and its own number
    const unsigned run = fdiv(rest, a.dParts), part = rest - run * a.dParts.d;
    const int h0 = run * kRun, mine = kRun == 1 ? 0 : g / a.G, own = kRun == 1 ? (int)part * 8 + g : g - mine * a.G;
    const bool real = mine < kRun && own < a.G && h0 + mine < a.c.Hkv;
    const int head = (h0 + mine) * a.G + own;
    uint4 qa = make_uint4(0, 0, 0, 0), qb = qa;
    if (real) {
        const uint4* row = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + n * a.q_token +
                                                          head * a.q_head);
        qa = row[t];
        qb = row[t + 4];
    }
    const int* pages = a.c.table + (size_t)max(seq, 0) * a.c.pages_per_seq;
    const bool padding = pos < 0 || seq < 0;
    bool bad = !padding && seq >= a.c.seqs, turned = false;
    float m = -INFINITY, l = 0.f, sc = 0.f, acc[8][4];
    unsigned qf[4][4];                                 // four products of 16 dims: (half, half of the dims)
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
    for (int r0 = 0; r0 < (kMany ? a.r.total : 1) && !padding && !bad; r0 += 32) {
        const RowOf row = row_of(a.r, r0 + lane);
        const unsigned live = __ballot_sync(kAll, r0 + lane < a.r.total && pos >= row.need);
        if (!live) continue;
        const bool lives = live >> lane & 1u;
        int slot;
        unsigned place = 0;
        bool found = slot_of<kTree>(a, n, pos, row.distance, lives, slot);
        if (found && lives) found = locate(a.c, pages, slot, place);
        bad = __any_sync(kAll, !found);
        if (bad) break;
        // a row that is not read stands for one that is: its score counts for nothing
        const unsigned some = __shfl_sync(kAll, place, __ffs(live) - 1);
        if (!lives) place = some;
        Places at;
#pragma unroll
        for (int i = 0; i < 4; ++i) at.k[i] = __shfl_sync(kAll, place, 8 * i + g);
#pragma unroll
        for (int i = 0; i < 8; ++i) at.v[i] = __shfl_sync(kAll, place, value_row(i, t));
        // the warp's key/value heads, keys of all and then values of all, two parts under way
        Part b[2];
        auto load = [&](int item) {
            const unsigned h = (unsigned)min(h0 + item % kRun, a.c.Hkv - 1) * a.c.head_stride;
            if (item < kRun) load_keys(a, at, h, t, b[item & 1]);
            else load_values(a, at, h, g, b[item & 1]);
        };
        load(0);
        load(1);
        if (!turned) {
            turned = true;
            rope_cs_f32(a.c.rope, lane, pos, turn[warp][0][lane], turn[warp][1][lane]);
            __syncwarp();
            float y[16];
            const unsigned w[8] = {qa.x, qa.y, qa.z, qa.w, qb.x, qb.y, qb.z, qb.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[2 * i] = __uint_as_float(w[i] << 16);
                y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
            float largest = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float cs = turn[warp][0][8 * t + i], sn = turn[warp][1][8 * t + i], u = y[i], v = y[8 + i];
                y[i] = u * cs - v * sn;
                y[8 + i] = v * cs + u * sn;
                largest = fmaxf(largest, fmaxf(fabsf(y[i]), fabsf(y[8 + i])));
            }
            float up, down;
            fit_half(mma::quad_max(largest), up, down);
            sc = down * a.scale;
#pragma unroll
            for (int s = 0; s < 4; ++s)                // dims 8t + 4 (s & 1) + 32 (s >> 1) + 0..3
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int d = 8 * (s >> 1) + 4 * (s & 1) + 2 * e;
                    const float y0 = y[d] * up, y1 = y[d + 1] * up;
                    const __half2 hi = __floats2half2_rn(y0, y1);
                    qf[s][2 * e] = *reinterpret_cast<const unsigned*>(&hi);
                    const float2 f = __half22float2(hi);
                    qf[s][2 * e + 1] = mma::pack_f16(y0 - f.x, y1 - f.y);
                }
        }
        float s[4][2];
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const Part& k = b[j & 1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float c[4];
                mma::mma_f16_16816_z(c, qf[0], k.x[2 * i].x, k.x[2 * i].y);
                mma::mma_f16_16816(c, qf[1], k.x[2 * i].z, k.x[2 * i].w);
                mma::mma_f16_16816(c, qf[2], k.x[2 * i + 1].x, k.x[2 * i + 1].y);
                mma::mma_f16_16816(c, qf[3], k.x[2 * i + 1].z, k.x[2 * i + 1].w);
                if (j == 0 || mine == j) {
                    s[i][0] = c[0] + c[2];
                    s[i][1] = c[1] + c[3];
                }
            }
            if (j + 2 < 2 * kRun) load(j + 2);
        }
        const unsigned pairs = __ballot_sync(kAll, row.pair);
        float weight[4][2], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + 2 * t;
            weight[i][0] = __shfl_sync(kAll, row.weight, r);
            weight[i][1] = __shfl_sync(kAll, row.weight, r + 1);
            s[i][0] *= sc * weight[i][0];
            s[i][1] *= sc * weight[i][1];
            if (pairs >> r & 1u) s[i][0] = s[i][1] = s[i][0] + s[i][1];
            if (!(live >> r & 1u)) s[i][0] = -INFINITY;
            if (!(live >> r & 2u)) s[i][1] = -INFINITY;
            top = fmaxf(top, fmaxf(s[i][0], s[i][1]));
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
        unsigned p[4][2];                              // [8 rows][upper, lower half]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = mma::ex2(s[i][0] - base) * weight[i][0], p1 = mma::ex2(s[i][1] - base) * weight[i][1];
            l += p0 + p1;
            p[i][0] = mma::pack_bf16(p0, p1);
            p[i][1] = mma::pack_bf16(p0 - __uint_as_float(p[i][0] << 16), p1 - __uint_as_float(p[i][0] & 0xffff0000u));
        }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const Part& v = b[(kRun + j) & 1];
            unsigned pj[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) pj[i] = kRun == 1 || mine == j ? p[i >> 1][i & 1] : 0u;
            if (!kMany && j == 0) add_values<true>(acc, pj, v.x);
            else add_values<false>(acc, pj, v.x);
            add_values<false>(acc, pj + 4, v.x + 4);
            if (kRun + j + 2 < 2 * kRun) load(kRun + j + 2);
        }
    }
    l = mma::quad_sum(l);
    float z = m + log2f(l), by = 1.f / l;
    if (padding) { by = 0.f; z = -INFINITY; }
    if (bad) by = z = NAN;
    if (real) {
        const size_t at = (size_t)n * a.H + head;
        uint4* out = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + at * kHeadDim + 16 * t);
        unsigned w[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = mma::pack_bf16((acc[2 * j][0] + acc[2 * j][2]) * by, (acc[2 * j + 1][0] + acc[2 * j + 1][2]) * by);
            w[4 + j] = mma::pack_bf16((acc[2 * j][1] + acc[2 * j][3]) * by, (acc[2 * j + 1][1] + acc[2 * j + 1][3]) * by);
        }
        out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        out[1] = make_uint4(w[4], w[5], w[6], w[7]);
        if (t == 0) a.lse[at] = z * kLn2;
    }
    if (bad && lane == 0) raise_status(a.status, kStatusPage);
}

template <int kRun, bool kMany>
cudaError_t launch(AttnArgs& a, cudaStream_t st) {
    const unsigned parts = (a.G + 7) / 8, runs = (a.c.Hkv + kRun - 1) / kRun;
    a.units = (unsigned)a.N * runs * parts;
    a.dRest = FastDiv::make(runs * parts);
    a.dParts = FastDiv::make(parts);
    const dim3 grid((a.units + kWarps - 1) / kWarps), block(32 * kWarps);
    return a.parents ? launch_kernel(attention_mma_kernel<kRun, kMany, true>, grid, block, 0, st, a)
                     : launch_kernel(attention_mma_kernel<kRun, kMany, false>, grid, block, 0, st, a);
}

}  // namespace

cudaError_t launch_attention_mma(const AttnArgs& args, cudaStream_t st) {
    AttnArgs a = args;
    // key/value heads of a warp: as many as its eight query heads allow, once that leaves
    // warps enough for the GPU
    const long long warps = (long long)a.N * a.c.Hkv;
    const long long most = std::min<long long>(std::min(8 / std::min(a.G, 8), a.c.Hkv), warps / (152 * 8));
    if (a.r.total > 32) return launch<1, true>(a, st);
    return most >= 8 ? launch<8, false>(a, st) : most >= 4 ? launch<4, false>(a, st)
           : most >= 2 ? launch<2, false>(a, st) : launch<1, false>(a, st);
}

}  // namespace cache
}  // namespace fibattn
