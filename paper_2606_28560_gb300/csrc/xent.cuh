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

// The fifth-generation tensor cores keep them as [segment][row] ...
cudaError_t launch_join_segments(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st);
// ... and the passes of few rows as [row][segment].
cudaError_t launch_join_rows(const Problem& p, const FwdParts& parts, int segments, float* loss, float* lse, cudaStream_t st);
// dx from parts [ranges][N][D].
cudaError_t launch_join_dx(const Problem& p, const float* parts, int ranges, void* dx, bool bf16, cudaStream_t st);

// One to four rows, as vectors (xent_stream.cu).  Scratch of the gradient: parts [blocks][N][D].
bool stream_applies(int N, int D);
int stream_segments(int V);
cudaError_t launch_stream(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st);
int stream_blocks(int V);
cudaError_t launch_stream_gradient(const Problem& p, const float* lse, const float* dloss, void* dx, void* dw, float* parts, int blocks,
                                   bool bf16, cudaStream_t st);

// Few rows (xent_rows.cu).  Scratch of the gradient: gradient [V][tokens], parts
// [ranges][N][D]; all fp32.
bool few_rows_applies(int N);
int few_rows_tokens(int N);                        // N rounded up to 8, 16 or 32
int few_rows_segments(int N, int D, int V);
cudaError_t launch_few_rows(const Problem& p, const FwdParts& parts, int segments, bool bf16, cudaStream_t st);
int few_rows_ranges(int N, int D, int V, bool bf16);
cudaError_t launch_few_rows_gradient(const Problem& p, const float* lse, const float* dloss, void* dx, void* dw, float* gradient,
                                     float* parts, int ranges, bool bf16, cudaStream_t st);

}  // namespace xent
}  // namespace fibattn
