// cache_api.cu -- argument checks and launches of the paged cache and of the
// attention over it (include/fibattn.h, "Generating with the attention").
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../../include/fibattn.h"
#include "cache.cuh"

using namespace fibattn;

namespace {

constexpr unsigned kReady = 0xf1bac4e1u;
constexpr long long kMaxSlots = 1LL << 30;           // storage slots of a sequence

bool misaligned16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
bool misaligned4(const void* a, const void* b, const void* c, const void* d) {
    return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) & 3u) != 0;
}

int launch_failed(cudaError_t e, const char* what) {
    return set_errorf(FIBATTN_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

int check_cache(const fibattn_cache* c) {
    if (!c || c->ready != kReady)
        return set_error(FIBATTN_ERR_INVALID_ARG, "the cache was not set up by fibattn_cache_init");
    return FIBATTN_OK;
}

cache::View view_of(const fibattn_cache& c) {
    cache::View v;
    v.k = c.k_pages;
    v.v = c.v_pages;
    v.table = c.table;
    v.page_stride = (unsigned)(c.page_stride / kHeadDim);
    v.row_stride = (unsigned)(c.row_stride / kHeadDim);
    v.head_stride = (unsigned)(c.head_stride / kHeadDim);
    v.pages = c.pages;
    v.Hkv = c.Hkv;
    v.seqs = c.seqs;
    v.pages_per_seq = c.pages_per_seq;
    v.dRows = FastDiv::make((unsigned)c.page_rows);
    std::memcpy(v.rope.F, c.phase, sizeof(v.rope.F));
    return v;
}

// Strides of a tensor of tokens, in elements: rows start on 16 bytes.
bool strides_ok(const fibattn_cache& c, long long token, long long head) {
    const long long unit = c.dtype == FIBATTN_BF16 ? 8 : 4;
    return token >= 0 && head >= 0 && token % unit == 0 && head % unit == 0;
}

int attention(const fibattn_cache* c, const void* q, long long q_token, long long q_head, void* out, float* lse,
              const int* positions, const int* parents, const int* slots, const int* seqs, int N, int H, int W,
              float alpha, const float* offsets, int K, const fibattn_opts* o, void* stream) {
    int rc = check_cache(c);
    if (rc) return rc;
    if (N < 0) return set_errorf(FIBATTN_ERR_INVALID_ARG, "N must not be negative (got %d)", N);
    if (H < 1 || H % c->Hkv || (long long)N * H > INT_MAX)
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "H (%d) must be a multiple of the cache's Hkv (%d) and N * H below 2^31",
                          H, c->Hkv);
    if (W < 0 || W > kMaxWindow) return set_errorf(FIBATTN_ERR_INVALID_ARG, "W must be in [0, %d] (got %d)", kMaxWindow, W);
    if (K < 0 || K > kMaxRungs) return set_errorf(FIBATTN_ERR_INVALID_ARG, "K must be in [0, %d] (got %d)", kMaxRungs, K);
    if (o && (o->rope_base != 0.f || o->Hkv || o->fwd_kernel || o->bwd_kernel || o->rotated_k || o->residuals))
        return set_error(FIBATTN_ERR_INVALID_ARG, "of the options only scale, no_dedup and round_offsets apply to a cache");
    const float scale = o && o->scale > 0.f ? o->scale : 0.125f;
    if (!std::isfinite(scale)) return set_error(FIBATTN_ERR_INVALID_ARG, "scale must be finite");
    RungParams r;
    // Every rung is kept, whatever the table reaches: the order of a query's rows, and with it the
    // last bits of its sums, then does not depend on the table's width.
    const int reach = INT_MAX - 127;                 // (the last one below a value of fp32 that fits an int)
    if ((rc = prepare_rungs(alpha, offsets, K, W, !(o && o->no_dedup), reach, &r, o && o->round_offsets))) return rc;
    if (N == 0) return FIBATTN_OK;
    if (!q || !out || !lse || !positions || (parents && !slots))
        return set_error(FIBATTN_ERR_INVALID_ARG, "NULL tensor pointer");
    if (misaligned4(positions, parents, slots, seqs))
        return set_error(FIBATTN_ERR_INVALID_ARG, "positions, parents, slots and seqs must be 4-byte aligned");
    if (misaligned16(q) || misaligned16(out) || ((uintptr_t)lse & 3u) || !strides_ok(*c, q_token, q_head))
        return set_error(FIBATTN_ERR_INVALID_ARG,
                         "tensor pointers must be 16-byte aligned (lse: 4-byte), strides multiples of 16 bytes");
    cache::AttnArgs a;
    std::memset(&a, 0, sizeof(a));
    a.c = view_of(*c);
    a.q = q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.out = out;
    a.lse = lse;
    a.positions = positions;
    a.seqs = seqs;
    a.parents = parents;
    a.slots = slots;
    a.N = N;
    a.H = H;
    a.G = H / c->Hkv;
    a.scale = scale * 1.4426950408889634f;
    int n = 0;
    for (int two = 1; two >= 0; --two)
        for (int k = 0; k < K; ++k)
            if ((r.active >> k & 1u) && (r.w[k] > 0.f) == (two == 1)) {
                a.r.near[n] = r.s0[k];
                a.r.far[n++] = r.w[k];
                ++(two ? a.r.pairs : a.r.singles);
            }
    a.r.window = W + 1;
    a.r.total = 2 * a.r.pairs + a.r.singles + a.r.window;
    if ((rc = device_status_word(&a.status))) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope p(parents ? "tree_fwd" : "cached_fwd", st);
    const cudaError_t e = c->dtype == FIBATTN_BF16 ? cache::launch_attention_mma(a, st) : cache::launch_attention_f32(a, st);
    return e == cudaSuccess ? FIBATTN_OK : launch_failed(e, "attention over the cache");
}

}  // namespace

extern "C" {

int fibattn_cache_init(fibattn_cache* c, void* k_pages, void* v_pages, int pages, int page_rows, int Hkv, int D,
                       long long page_stride, long long row_stride, long long head_stride,
                       const int* table, int seqs, int pages_per_seq, int dtype, float rope_base) {
    if (!c) return set_error(FIBATTN_ERR_INVALID_ARG, "NULL cache");
    c->ready = 0;
    if (dtype != FIBATTN_F32 && dtype != FIBATTN_BF16) return set_errorf(FIBATTN_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (D != kHeadDim) return set_errorf(FIBATTN_ERR_UNSUPPORTED, "only D == %d is built (got %d)", kHeadDim, D);
    if (pages < 1 || page_rows < 1 || Hkv < 1 || seqs < 1 || pages_per_seq < 1)
        return set_error(FIBATTN_ERR_INVALID_ARG, "pages, page_rows, Hkv, seqs and pages_per_seq must be at least 1");
    if ((long long)page_rows * pages_per_seq > kMaxSlots)
        return set_error(FIBATTN_ERR_INVALID_ARG, "page_rows * pages_per_seq must be at most 2^30");
    if (!k_pages || !v_pages || !table) return set_error(FIBATTN_ERR_INVALID_ARG, "NULL pool or table pointer");
    if (((uintptr_t)k_pages & 31u) || ((uintptr_t)v_pages & 31u) || ((uintptr_t)table & 3u))
        return set_error(FIBATTN_ERR_INVALID_ARG, "pool pointers must be 32-byte aligned (table: 4-byte)");
    const long long strides[3] = {page_stride, row_stride, head_stride}, sizes[3] = {pages, page_rows, Hkv};
    long long last = 0;                              // the last row of the pool, counted in rows of 64
    for (int i = 0; i < 3; ++i) {
        if (strides[i] < kHeadDim || strides[i] % kHeadDim)
            return set_error(FIBATTN_ERR_INVALID_ARG, "pool strides must be positive multiples of 64 elements");
        const long long rows = strides[i] / kHeadDim;
        if (rows >= 1LL << 32 || (last += (sizes[i] - 1) * rows) >= 1LL << 32)
            return set_error(FIBATTN_ERR_INVALID_ARG, "the pool's rows must lie within 2^32 rows of 64 elements");
    }
    if (rope_base == 0.f) rope_base = 1e4f;
    if (!(rope_base > 1.f) || !std::isfinite(rope_base))
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "rope_base must be finite and > 1 (got %g)", (double)rope_base);
    c->k_pages = k_pages;
    c->v_pages = v_pages;
    c->table = table;
    c->page_stride = page_stride;
    c->row_stride = row_stride;
    c->head_stride = head_stride;
    c->pages = pages;
    c->page_rows = page_rows;
    c->Hkv = Hkv;
    c->seqs = seqs;
    c->pages_per_seq = pages_per_seq;
    c->dtype = dtype;
    RopeParams rope;
    prepare_rope(rope_base, &rope);
    std::memcpy(c->phase, rope.F, sizeof(c->phase));
    c->ready = kReady;
    return FIBATTN_OK;
}

int fibattn_cache_append(const fibattn_cache* c, const void* k, long long k_token_stride, long long k_head_stride,
                         const void* v, long long v_token_stride, long long v_head_stride,
                         const int* positions, const int* slots, const int* seqs, int N, void* stream) {
    int rc = check_cache(c);
    if (rc) return rc;
    if (N < 0 || (long long)N * c->Hkv > INT_MAX)
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "N must not be negative and N * Hkv below 2^31 (got N %d)", N);
    if (N == 0) return FIBATTN_OK;
    if (!k || !v || !positions) return set_error(FIBATTN_ERR_INVALID_ARG, "NULL tensor pointer");
    if (misaligned4(positions, slots, seqs, nullptr))
        return set_error(FIBATTN_ERR_INVALID_ARG, "positions, slots and seqs must be 4-byte aligned");
    if (misaligned16(k) || misaligned16(v) || !strides_ok(*c, k_token_stride, k_head_stride) ||
        !strides_ok(*c, v_token_stride, v_head_stride))
        return set_error(FIBATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned, strides multiples of 16 bytes");
    cache::AppendArgs a;
    std::memset(&a, 0, sizeof(a));
    a.c = view_of(*c);
    a.k = k;
    a.v = v;
    a.k_token = k_token_stride;
    a.k_head = k_head_stride;
    a.v_token = v_token_stride;
    a.v_head = v_head_stride;
    a.positions = positions;
    a.slots = slots;
    a.seqs = seqs;
    a.N = N;
    if ((rc = device_status_word(&a.status))) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ProfScope p("cache_append", st);
    const cudaError_t e = cache::launch_append(a, c->dtype == FIBATTN_BF16, st);
    return e == cudaSuccess ? FIBATTN_OK : launch_failed(e, "append to the cache");
}

int fibattn_cached_fwd(const fibattn_cache* c, const void* q, long long q_token_stride, long long q_head_stride,
                       void* out, float* lse, const int* positions, const int* seqs, int N, int H, int W,
                       float alpha, const float* offsets, int K, const fibattn_opts* opts, void* stream) {
    return attention(c, q, q_token_stride, q_head_stride, out, lse, positions, nullptr, nullptr, seqs, N, H, W, alpha,
                     offsets, K, opts, stream);
}

int fibattn_tree_fwd(const fibattn_cache* c, const void* q, long long q_token_stride, long long q_head_stride,
                     void* out, float* lse, const int* positions, const int* parents, const int* slots,
                     const int* seqs, int N, int H, int W,
                     float alpha, const float* offsets, int K, const fibattn_opts* opts, void* stream) {
    if (N > 0 && !parents) return set_error(FIBATTN_ERR_INVALID_ARG, "NULL tensor pointer");
    return attention(c, q, q_token_stride, q_head_stride, out, lse, positions, parents, slots, seqs, N, H, W, alpha,
                     offsets, K, opts, stream);
}

}  // extern "C"
