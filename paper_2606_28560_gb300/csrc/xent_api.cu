// xent_api.cu -- argument checks, workspace layout and launches of the linear
// cross entropy (include/fibattn.h).
#include <algorithm>
#include <cstdint>

#include "../../include/fibattn.h"
#include "xent_mma.cuh"

using namespace fibattn;

namespace {

bool misaligned16(const void* p) { return ((uintptr_t)p & 15u) != 0; }

int check_sizes(int N, int D, int V, int dtype) {
    if (dtype != FIBATTN_F32 && dtype != FIBATTN_BF16) return set_errorf(FIBATTN_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (N < 0 || N > (1 << 24)) return set_errorf(FIBATTN_ERR_INVALID_ARG, "N must be in [0, 2^24] (got %d)", N);
    if (D < 1 || D > 8192) return set_errorf(FIBATTN_ERR_INVALID_ARG, "D must be in [1, 8192] (got %d)", D);
    if (V < 1 || V > (1 << 24)) return set_errorf(FIBATTN_ERR_INVALID_ARG, "V must be in [1, 2^24] (got %d)", V);
    return FIBATTN_OK;
}

int launch_failed(cudaError_t e, const char* what) {
    return set_errorf(FIBATTN_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

size_t fibattn_linear_xent_fwd_workspace_bytes(int N, int D, int V, int dtype) {
    if (check_sizes(N, D, V, dtype)) return 0;
    return xent::plan_forward(N, D, V, dtype == FIBATTN_BF16).total;
}

int fibattn_linear_xent_fwd(const void* x, const void* w, const long long* targets, float* loss, float* lse,
                            int N, int D, int V, long long ignore_index, int dtype,
                            void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(N, D, V, dtype);
    if (rc) return rc;
    if (N == 0) return FIBATTN_OK;
    if (!x || !w || !targets || !loss || !lse || !workspace)
        return set_error(FIBATTN_ERR_INVALID_ARG, "NULL tensor or workspace pointer");
    if (misaligned16(x) || misaligned16(w) || misaligned16(loss) || misaligned16(lse) || misaligned16(workspace) ||
        ((uintptr_t)targets & 7u))
        return set_error(FIBATTN_ERR_INVALID_ARG, "pointers must be 16-byte aligned (targets: 8-byte)");
    const bool bf16 = dtype == FIBATTN_BF16;
    const xent::FwdPlan plan = xent::plan_forward(N, D, V, bf16);
    if (workspace_bytes < plan.total)
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "workspace too small: %zu < %zu", workspace_bytes, plan.total);
    xent::Problem p{x, w, targets, N, D, V, ignore_index, nullptr};
    if ((rc = bind_device_context())) return rc;
    if ((rc = device_status_word(&p.status))) return rc;
    const cudaError_t e = xent::run_forward(p, plan, static_cast<char*>(workspace), bf16, loss, lse,
                                            static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? FIBATTN_OK : launch_failed(e, "cross-entropy forward");
}

size_t fibattn_linear_xent_bwd_workspace_bytes(int N, int D, int V, int dtype) {
    if (check_sizes(N, D, V, dtype)) return 0;
    return xent::plan_backward(N, D, V, dtype == FIBATTN_BF16).total;
}

int fibattn_linear_xent_bwd(const void* x, const void* w, const long long* targets, const float* lse, const float* dloss,
                            void* dx, void* dw, int N, int D, int V, long long ignore_index, int dtype,
                            void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(N, D, V, dtype);
    if (rc) return rc;
    if (N > 0 && ((!dx && !dw) || !x || !w || !targets || !lse || !dloss || !workspace))
        return set_error(FIBATTN_ERR_INVALID_ARG, "NULL tensor or workspace pointer");
    if (misaligned16(x) || misaligned16(w) || misaligned16(lse) || misaligned16(dloss) || misaligned16(dx) ||
        misaligned16(dw) || misaligned16(workspace) || ((uintptr_t)targets & 7u))
        return set_error(FIBATTN_ERR_INVALID_ARG, "pointers must be 16-byte aligned (targets: 8-byte)");
    const bool bf16 = dtype == FIBATTN_BF16;
    const xent::BwdPlan plan = xent::plan_backward(N, D, V, bf16);
    if (N > 0 && workspace_bytes < plan.total)
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "workspace too small: %zu < %zu", workspace_bytes, plan.total);
    xent::Problem p{x, w, targets, N, D, V, ignore_index, nullptr};
    if ((rc = bind_device_context())) return rc;
    if ((rc = device_status_word(&p.status))) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (N == 0) {                                // no rows: the head's gradient is zero
        e = dw ? cudaMemsetAsync(dw, 0, (size_t)V * D * (bf16 ? 2 : 4), st) : cudaSuccess;
        return e == cudaSuccess ? FIBATTN_OK : launch_failed(e, "zero gradients of an empty batch");
    }
    e = xent::run_backward(p, plan, static_cast<char*>(workspace), bf16, lse, dloss, dx, dw, st);
    return e == cudaSuccess ? FIBATTN_OK : launch_failed(e, "cross-entropy backward");
}

}  // extern "C"
