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

// Per-row statistics of the forward: for each segment of the columns the
// maximum of the logits and the sum of exp(logit - maximum); target_logit[n] is
// written by whoever forms that logit.
struct FwdParts {
    float* m;
    float* l;
    float* target_logit;
};

// The tensor-core forward keeps them as [segment][row] ...
cudaError_t launch_join_segments(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st);
// ... the forward of few rows as [row][segment].
int few_rows_segments(int V);
cudaError_t launch_few_rows(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st);
cudaError_t launch_join_rows(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st);

// The gradient of few rows: parts is [blocks][N][D] fp32 of scratch.
int few_rows_at_most(int N, int D);                // rows that it can take, of N
int few_rows_blocks(int V);
cudaError_t launch_few_rows_gradient(const Problem& p, const float* lse, const float* dloss, void* dx, void* dw, float* parts,
                                     int blocks, bool bf16, cudaStream_t st);

}  // namespace xent
}  // namespace fibattn
