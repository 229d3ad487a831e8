// xent.cuh -- shared definitions of the linear cross-entropy kernels (not part
// of the C ABI; the calls are declared in include/fibattn.h).
#pragma once
#include "fibattn_internal.cuh"

namespace fibattn {
namespace xent {

struct Problem {
    const void* x;             // [N][D]
    const void* w;             // [V][D]
    const long long* targets;  // [N]
    int N, D, V;
    long long ignore_index;
    unsigned* status;
};

// What row n's target says: its column, or kIgnored / kBad (no column is ever
// equal to either).
constexpr int kIgnored = -1, kBad = -2;
__device__ __forceinline__ int target_column(const Problem& p, int n) {
    const long long t = p.targets[n];
    if (t == p.ignore_index) return kIgnored;
    return (t >= 0 && t < p.V) ? (int)t : kBad;
}

// Per-row partials of the forward: segment s of row n holds the maximum of the
// logits it covers at m[s * N + n] and the sum of exp(logit - m) at
// l[s * N + n]; target_logit[n] is written by whoever forms that logit.
struct FwdParts {
    float* m;
    float* l;
    float* target_logit;
};

cudaError_t launch_fwd_simple(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st);
int fwd_simple_segments(int N, int V);
cudaError_t launch_combine(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse,
                           cudaStream_t st);

// Backward, columns [v0, v0 + cols) of the vocabulary: g (fp32, row length
// ldg) and then its two products.  dx_acc: fp32 [N][D], holds the sum over the
// earlier pieces unless `first`; the `last` piece writes dx.
cudaError_t launch_grad_simple(const Problem& p, const float* lse, const float* dloss, float* g, int ldg, int v0,
                               int cols, bool bf16, cudaStream_t st);
cudaError_t launch_products_simple(const Problem& p, const float* g, int ldg, int v0, int cols, bool first, bool last,
                                   float* dx_acc, void* dx, void* dw, bool bf16, cudaStream_t st);

}  // namespace xent
}  // namespace fibattn
