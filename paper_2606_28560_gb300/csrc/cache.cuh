// cache.cuh -- the paged cache of keys and values on the device, shared by the
// append and the attention kernels (include/fibattn.h, "Generating with the
// attention").
#pragma once

#include "fibattn_internal.cuh"

namespace fibattn {
namespace cache {

constexpr int kMaxRows = 2 * kMaxRungs + kMaxWindow + 1;   // cache rows of one query

// Offsets are counted in rows of 64 elements: 32 bits then reach 2^32 rows, more
// than fit a GPU (half a terabyte of 16-bit rows).
struct View {
    void* k;
    void* v;
    const int* table;
    unsigned page_stride, row_stride, head_stride;   // rows
    int pages, Hkv, seqs, pages_per_seq;
    FastDiv dRows;                                   // by the rows of a page
    RopeParams rope;
};

struct AppendArgs {
    View c;
    const void* k;
    const void* v;
    long long k_token, k_head, v_token, v_head;      // strides in elements
    const int* positions;
    const int* slots;                                // or nullptr: positions
    const int* seqs;                                 // or nullptr: token n is sequence n
    int N;
    int per;                                         // tokens of a warp
    unsigned* status;
};

// The cache rows of a query, in the order they are read: the interpolated rungs,
// two rows each (floor, far), then rungs at integer distances, then the window.
struct Rows {
    int pairs, singles, window;                      // rungs of two rows, of one row; W + 1
    int total;                                       // 2 pairs + singles + window
    int near[kMaxRungs];                             // floor(d_k): of the pairs, then of the singles
    float far[kMaxRungs];                            // weight of the far row
};

struct AttnArgs {
    View c;
    const void* q;
    long long q_token, q_head;                       // strides in elements
    void* out;
    float* lse;
    const int* positions;
    const int* seqs;
    const int* parents;                              // trees only
    const int* slots;
    int N, H, G;                                     // G = H / Hkv query heads per key/value head
    int run;                                         // of a warp: key/value heads (bf16), query heads (fp32)
    unsigned units;                                  // warps
    FastDiv dRest, dParts;                           // by the warps of a token, by the parts of a group
    float scale;                                     // times log2 e: softmax in base 2
    Rows r;
    unsigned* status;
};

cudaError_t launch_append(const AppendArgs& a, bool bf16, cudaStream_t st);
cudaError_t launch_attention_f32(const AttnArgs& a, cudaStream_t st);
cudaError_t launch_attention_mma(const AttnArgs& a, cudaStream_t st);          // bf16

// cos and sin of the angle of pair m at position pos, to fp32 rounding: the phase is
// an integer fraction of a turn (RopeParams), cut to 2^-32 of one (1.5e-9 in the
// angle); its quadrant is taken off exactly, and rounding what is left, at most an
// eighth of a turn, costs 2^-24 of it.  rope_cs, with 2^-21, would show in fp32 keys.
__device__ __forceinline__ void rope_cs_f32(const RopeParams& rp, int m, int pos, float& c, float& s) {
    const unsigned turn = (unsigned)(((unsigned long long)(unsigned)pos * rp.F[m]) >> 32);   // of 2^32
    const unsigned quarter = (turn + (1u << 29)) >> 30;
    const float x = (float)(int)(turn - (quarter << 30)) * 4.6566128730773926e-10f;          // half turns
    float cs, sn;
    sincospif(x, &sn, &cs);
    const float a = (quarter & 1) ? sn : cs, b = (quarter & 1) ? cs : sn;
    c = ((quarter + 1) & 2) ? -a : a;
    s = (quarter & 2) ? -b : b;
}

// The row of storage slot `slot` of the sequence whose table row is `pages`; false
// if there is none.
__device__ __forceinline__ bool locate(const View& c, const int* pages, int slot, unsigned& row) {
    if (slot < 0) return false;
    const unsigned p = fdiv((unsigned)slot, c.dRows);
    if (p >= (unsigned)c.pages_per_seq) return false;
    const int page = pages[p];
    if ((unsigned)page >= (unsigned)c.pages) return false;
    row = (unsigned)page * c.page_stride + ((unsigned)slot - p * c.dRows.d) * c.row_stride;
    return true;
}

}  // namespace cache
}  // namespace fibattn
