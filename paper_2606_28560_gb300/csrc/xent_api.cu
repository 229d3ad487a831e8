// xent_api.cu -- argument checks, workspace layout and launches of the linear
// cross entropy (include/fibattn.h).
#include <algorithm>
#include <cstdint>

#include "../../include/fibattn.h"
#include "xent.cuh"

using namespace fibattn;

namespace {

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
bool misaligned16(const void* p) { return ((uintptr_t)p & 15u) != 0; }

int check_sizes(int N, int D, int V, int dtype) {
    if (dtype != FIBATTN_F32 && dtype != FIBATTN_BF16) return set_errorf(FIBATTN_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (N < 0 || N > (1 << 24)) return set_errorf(FIBATTN_ERR_INVALID_ARG, "N must be in [0, 2^24] (got %d)", N);
    if (D < 1 || D > 8192) return set_errorf(FIBATTN_ERR_INVALID_ARG, "D must be in [1, 8192] (got %d)", D);
    if (V < 1 || V > (1 << 24)) return set_errorf(FIBATTN_ERR_INVALID_ARG, "V must be in [1, 2^24] (got %d)", V);
    return FIBATTN_OK;
}

struct FwdLayout {
    int segments;
    size_t m, l, target, total;
};

FwdLayout fwd_layout(int N, int D, int V, int dtype) {
    FwdLayout L;
    L.segments = xent::fwd_simple_segments(N, V);
    size_t off = 0;
    L.m = off; off += up256((size_t)L.segments * N * 4);
    L.l = off; off += up256((size_t)L.segments * N * 4);
    L.target = off; off += up256((size_t)N * 4);
    L.total = off;
    return L;
}

// The piece of the vocabulary that the backward takes at a time: g of it is
// at most 256 MiB (at least 128 columns).
struct BwdLayout {
    int cols;                  // columns of a piece
    size_t g, dx_acc, total;
};

BwdLayout bwd_layout(int N, int D, int V, int dtype) {
    BwdLayout L;
    const long long fit = (256ll << 20) / (4ll * std::max(N, 1)) / 128 * 128;
    L.cols = (int)std::min<long long>((V + 3) / 4 * 4, std::max(128ll, fit));
    size_t off = 0;
    L.g = off; off += up256((size_t)N * L.cols * 4);
    L.dx_acc = off; off += up256((size_t)N * D * 4);
    L.total = off;
    return L;
}

int launch_failed(cudaError_t e, const char* what) {
    return set_errorf(FIBATTN_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

size_t fibattn_linear_xent_fwd_workspace_bytes(int N, int D, int V, int dtype) {
    if (check_sizes(N, D, V, dtype)) return 0;
    return fwd_layout(N, D, V, dtype).total;
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
    const FwdLayout L = fwd_layout(N, D, V, dtype);
    if (workspace_bytes < L.total)
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "workspace too small: %zu < %zu", workspace_bytes, L.total);
    xent::Problem p{x, w, targets, N, D, V, ignore_index, nullptr};
    if ((rc = bind_device_context())) return rc;
    if ((rc = device_status_word(&p.status))) return rc;
    char* ws = static_cast<char*>(workspace);
    const xent::FwdParts parts{reinterpret_cast<float*>(ws + L.m), reinterpret_cast<float*>(ws + L.l),
                               reinterpret_cast<float*>(ws + L.target)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == FIBATTN_BF16;
    cudaError_t e;
    {
        ProfScope s("xent_fwd", st);
        e = xent::launch_fwd_simple(p, parts, L.segments, bf16, st);
    }
    if (e != cudaSuccess) return launch_failed(e, "cross-entropy forward launch");
    {
        ProfScope s("xent_combine", st);
        e = xent::launch_combine(p, parts, L.segments, loss, lse, st);
    }
    if (e != cudaSuccess) return launch_failed(e, "cross-entropy combine launch");
    return FIBATTN_OK;
}

size_t fibattn_linear_xent_bwd_workspace_bytes(int N, int D, int V, int dtype) {
    if (check_sizes(N, D, V, dtype)) return 0;
    return bwd_layout(N, D, V, dtype).total;
}

int fibattn_linear_xent_bwd(const void* x, const void* w, const long long* targets, const float* lse, const float* dloss,
                            void* dx, void* dw, int N, int D, int V, long long ignore_index, int dtype,
                            void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(N, D, V, dtype);
    if (rc) return rc;
    if (!dw || (N > 0 && (!x || !w || !targets || !lse || !dloss || !dx || !workspace)))
        return set_error(FIBATTN_ERR_INVALID_ARG, "NULL tensor or workspace pointer");
    if (misaligned16(x) || misaligned16(w) || misaligned16(lse) || misaligned16(dloss) || misaligned16(dx) ||
        misaligned16(dw) || misaligned16(workspace) || ((uintptr_t)targets & 7u))
        return set_error(FIBATTN_ERR_INVALID_ARG, "pointers must be 16-byte aligned (targets: 8-byte)");
    const BwdLayout L = bwd_layout(N, D, V, dtype);
    if (N > 0 && workspace_bytes < L.total)
        return set_errorf(FIBATTN_ERR_INVALID_ARG, "workspace too small: %zu < %zu", workspace_bytes, L.total);
    xent::Problem p{x, w, targets, N, D, V, ignore_index, nullptr};
    if ((rc = bind_device_context())) return rc;
    if ((rc = device_status_word(&p.status))) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == FIBATTN_BF16;
    cudaError_t e;
    if (N == 0) {                                // no rows: the head's gradient is zero
        e = cudaMemsetAsync(dw, 0, (size_t)V * D * (bf16 ? 2 : 4), st);
        return e == cudaSuccess ? FIBATTN_OK : launch_failed(e, "zero gradients of an empty batch");
    }
    char* ws = static_cast<char*>(workspace);
    float* g = reinterpret_cast<float*>(ws + L.g);
    float* dx_acc = reinterpret_cast<float*>(ws + L.dx_acc);
    for (int v0 = 0; v0 < V; v0 += L.cols) {
        const int cols = std::min(L.cols, V - v0);
        {
            ProfScope s("xent_grad", st);
            e = xent::launch_grad_simple(p, lse, dloss, g, L.cols, v0, cols, bf16, st);
        }
        if (e != cudaSuccess) return launch_failed(e, "cross-entropy gradient launch");
        {
            ProfScope s("xent_products", st);
            e = xent::launch_products_simple(p, g, L.cols, v0, cols, v0 == 0, v0 + cols >= V, dx_acc, dx, dw, bf16, st);
        }
        if (e != cudaSuccess) return launch_failed(e, "cross-entropy product launch");
    }
    return FIBATTN_OK;
}

}  // extern "C"
