/*
 * fibattn.h -- C ABI of the GB300 (sm_103a) library for depth-staggered
 * scaled-Fibonacci sparse attention (arXiv 2606.28560).
 *
 * The operation (Section 2, "Attended set"): query i attends to the dense
 * causal window at distances 0..W plus K rungs at continuous distances
 * d_k = alpha * f_k.  A rung is read by linear interpolation between the
 * floor and floor-plus-one positions; RoPE is applied to q and k at their true
 * positions before the gather; the attended scores go through a softmax and
 * weight the (equally interpolated) values.  alpha = 0.5 + sigmoid(theta) is
 * one scalar per layer (Section 2, "The per-layer scalar").
 *
 * Conventions shared by every call:
 *   - Tensor layouts are row-major and contiguous: q, out, dout, dq are
 *     [B][H][T][D]; k, v, dk, dv are [B][Hkv][T][D]; lse is [B][H][T] fp32.
 *     Element type is given by `dtype` (fp32 or bf16); lse is always fp32.
 *   - Tensor, workspace and output-scalar pointers are DEVICE pointers owned by
 *     the caller and aligned to 16 bytes.  `offsets` is a HOST array of K floats
 *     (the base sequence f_k, e.g. 1,2,3,5,...,987) read during the call only.
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy default stream).
 *     Device work is asynchronous on that stream; a call returns after launch.
 *     Work goes to the calling thread's current device; a compute call makes
 *     that device's primary context current on the thread if none is.
 *   - Return value is a fibattn_status.  Argument errors are reported before
 *     any launch.  Faults raised asynchronously by the device surface at the
 *     caller's next synchronisation.  fibattn_last_error() gives a thread-local
 *     message for the last non-OK status.  No C++ exception crosses the ABI.
 *   - Limits: D == 64; 0 <= W <= 1024; 0 <= K <= 32; 1 <= T <= 2^20;
 *     0.5 <= alpha <= 1.5; every d_k = fl32(alpha * f_k) must be finite and
 *     >= 0; H % Hkv == 0.
 *   - Readings of the paper taken where it is silent: scale = 1/sqrt(D); the
 *     floor is taken of the distance, the far row i-floor(d)-1 has weight
 *     d-floor(d); a rung with d_k > i is masked; with dedup a rung with
 *     d_k <= W is dropped (the attended set is a set union); RoPE pairs
 *     dimension m with m+D/2 at frequency rope_base^(-2m/D).
 */
#ifndef FIBATTN_H
#define FIBATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FIBATTN_OK = 0,
    FIBATTN_ERR_INVALID_ARG = 1,   /* bad shape, pointer, alignment, alpha, ...   */
    FIBATTN_ERR_UNSUPPORTED = 2,   /* valid but not built (e.g. D != 64)           */
    FIBATTN_ERR_CUDA = 3,          /* a CUDA runtime call or launch failed         */
    FIBATTN_ERR_INTERNAL = 4,      /* an internal consistency check failed, or a
                                      kernel gave up a bounded wait (see
                                      fibattn_check_status)                        */
    FIBATTN_ERR_RANGE = 5          /* an operand left the range of the library's
                                      16-bit rotated rows, a target that of the
                                      vocabulary, or a page that of the pool
                                      (fibattn_check_status)                       */
} fibattn_status;

typedef enum { FIBATTN_F32 = 0, FIBATTN_BF16 = 1 } fibattn_dtype;

/* Options.  Zero-initialised fields take the defaults in brackets. */
typedef struct {
    float rope_base;   /* RoPE frequency base [1e4] (Section 3, "Model and training") */
    float scale;       /* score scale; <= 0 means 1/sqrt(D)                            */
    int   Hkv;         /* key/value heads (GQA); 0 means Hkv = H                       */
    int   no_dedup;    /* 0: drop rungs with d_k <= W [default]; 1: keep them          */
    int   fwd_kernel;  /* forward kernel: 0 automatic [default]; 1 row-gather kernel
                          (any W and K, fp32 or bf16); 3 tensor-core kernel (bf16
                          I/O, W <= 16, K <= 16); 2 is not built.
                          FIBATTN_ERR_UNSUPPORTED when the choice does not apply. */
    int   bwd_kernel;  /* backward query pass: 0 automatic [default]; 1 row-gather
                          single sweep (Delta accumulated from the slots, `out`
                          unused); 2 tensor-core kernel (bf16 I/O, `out` given,
                          W <= 16, K <= 16; FIBATTN_ERR_UNSUPPORTED otherwise).
                          Automatic takes 2 where it applies, else 1. */
    void* rotated_k;   /* optional device buffer of B*Hkv*T*D elements (fp16 for bf16
                          I/O, fp32 for fp32 I/O), 16-byte aligned [NULL].  Given
                          it, fibattn_fwd writes the RoPE-rotated keys there
                          instead of into its workspace, and fibattn_bwd reads
                          them from there instead of rotating k again (k may then
                          be NULL): a caller that keeps this buffer from the
                          forward to the backward keeps it in place of k. */
    void* residuals;   /* optional device buffer of fibattn_residual_bytes(...) bytes,
                          16-byte aligned [NULL].  Given it, fibattn_fwd also writes
                          what the backward would otherwise recompute from q and k:
                          the RoPE-rotated queries (bf16 [B][H][T][D]), the
                          unnormalised softmax weight exp(s - max) of every
                          slot (fp32 [B][H][S][T], S = W + 1 + K: window
                          distances 0..W, then rung k at W + 1 + k; 0 where not
                          attended; rungs that are never read -- dropped by
                          dedup or beyond T's reach -- are left unwritten), the
                          far-minus-floor raw score q~ . (k~_far - k~_floor) of
                          every rung (fp32 [B][H][K][T]) and 1 / (sum of the
                          weights) per query (fp32 [B][H][T]), so that the
                          probability is weight / sum; the four arrays follow
                          one another in
                          that order, each starting at the next multiple of 256
                          bytes.  Only the tensor-core forward writes them:
                          bf16 I/O, and fwd_kernel 0 or 3 with its layout applying;
                          otherwise fibattn_fwd fails with FIBATTN_ERR_UNSUPPORTED
                          before any launch.  fibattn_bwd given the buffer filled by
                          the forward of the same inputs and parameters reads them
                          in its tensor-core passes instead of recomputing the
                          scores; when its tensor-core passes do not apply it
                          ignores the buffer. */
    int   round_offsets; /* 0: continuous distances d_k = fl32(alpha f_k), rungs
                          interpolated [default]; 1: the integer-offset variants
                          (Section 2, "Implementation note", the fused
                          boolean-mask path): d_k rounded to the nearest integer,
                          ties to even, after the fp32 product; every rung then
                          reads one row.  fibattn_bwd then requires dtheta and dd
                          to be NULL (the rounded distances do not vary with
                          alpha). */
} fibattn_opts;

/* ---------------------------------------------------------------------------
 * Forward: out[b,h,i,:] and lse[b,h,i] (log of the softmax normaliser, in the
 * scaled-score domain) for every query (Section 2, "Attended set").
 * workspace: device scratch of at least fibattn_fwd_workspace_bytes(...)
 * bytes; contents on entry are ignored and on exit are unspecified.
 * out may not alias q, k, v or workspace.
 * ------------------------------------------------------------------------- */
size_t fibattn_fwd_workspace_bytes(int B, int H, int T, int D, int W, int K,
                                   int dtype, const fibattn_opts* opts);

int fibattn_fwd(const void* q, const void* k, const void* v,
                void* out, float* lse,
                int B, int H, int T, int D, int W,
                float alpha, const float* offsets, int K,
                int dtype, const fibattn_opts* opts,
                void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Backward (the chain rule of the forward definition; the paper trains every
 * model through this path, Section 2 "Implementation note").
 * Inputs: q, k, v, dout as above and lse from fibattn_fwd of the same inputs.
 * out: the output of that forward call, or NULL.  With out, the softmax term
 * Delta_i = sum_slots p dp (= dout_i . out_i) is read as dout_i . out_i, which
 * lets the tensor-core query pass (opts->bwd_kernel) form each score gradient
 * in one pass; without it Delta is accumulated from the slots.
 * Outputs (overwritten, not accumulated): dq [B,H,T,D], dk and dv [B,Hkv,T,D]
 * in `dtype`, gradients with respect to the pre-RoPE q and k; dtheta (device,
 * 1 float, may be NULL) = dL/dtheta with alpha = 0.5 + sigmoid(theta); dd
 * (device, K floats, may be NULL) = dL/dd_k for each rung distance.
 * dL/dalpha = sum_k f_k dd_k.  With both NULL (a fixed alpha schedule, alpha
 * not trained) the rung-distance gradient is not computed at all.
 * At an integer d_k the distance derivative is one-sided, from above.
 * dq, dk, dv, dtheta and dd may not alias each other, an input, the
 * residuals or the workspace.
 * ------------------------------------------------------------------------- */
size_t fibattn_bwd_workspace_bytes(int B, int H, int T, int D, int W, int K,
                                   int dtype, const fibattn_opts* opts);

int fibattn_bwd(const void* q, const void* k, const void* v,
                const void* out, const float* lse, const void* dout,
                void* dq, void* dk, void* dv, float* dtheta, float* dd,
                int B, int H, int T, int D, int W,
                float alpha, const float* offsets, int K,
                int dtype, const fibattn_opts* opts,
                void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of the forward residuals (fibattn_opts.residuals) for these sizes;
 * 0 for invalid sizes or fp32 I/O (no residuals). */
size_t fibattn_residual_bytes(int B, int H, int T, int D, int W, int K, int dtype);

/* Thread-local message for the last non-OK status returned on this thread. */
const char* fibattn_last_error(void);

/* ---------------------------------------------------------------------------
 * Device status (no counterpart in the paper).  Kernels report conditions
 * that no argument check can catch before launch into a per-device status
 * word, without stopping:
 *   bit 0 -- a kernel gave up waiting for one of its own shared-memory staging
 *            copies (each wait is bounded to 1 s of the GPU's global timer);
 *            the affected tiles' outputs (out, lse, gradients) are NaN.
 *   bit 1 -- an entry of a 16-bit rotated row reached 65520 in magnitude:
 *            the bf16 path keeps the RoPE-rotated keys, and the rotated
 *            queries times the score scale, in fp16 (for score precision),
 *            which cannot hold it.
 *   bit 2 -- fibattn_linear_xent_fwd or _bwd met a target outside [0, V) that
 *            is not ignore_index (that row's loss is NaN).
 *   bit 3 -- a call on a paged cache met a sequence, storage slot, page or
 *            parent that does not exist (see fibattn_cache_init).
 * fibattn_check_status synchronises `stream`, reads the calling thread's
 * current device's word into *flags (may be NULL) and clears it.  Returns
 * FIBATTN_ERR_INTERNAL if bit 0 was set, else FIBATTN_ERR_RANGE if bit 1, 2 or
 * 3 was set, else FIBATTN_OK.  Compute calls never synchronise to look at it.
 * ------------------------------------------------------------------------- */
int fibattn_check_status(void* stream, unsigned* flags);

/* Test hook for the bounded wait: launches one warp on `stream` that waits on
 * a shared-memory barrier no copy will complete, with a bound of timeout_us
 * microseconds (1 .. 1e7); the wait runs out and sets status bit 0, which a
 * following fibattn_check_status reports.  The kernel touches no memory but
 * its own shared barrier and the status word. */
int fibattn_test_wait_timeout(unsigned timeout_us, void* stream);

/* ---------------------------------------------------------------------------
 * Host-side parameter prep (no GPU needed).
 * ------------------------------------------------------------------------- */

/* Rung prep (Section 2): d[k] = fl32(alpha * f[k]) (with round_offsets then
 * rounded to the nearest integer, ties to even); s0[k] = floor(d[k]);
 * w[k] = d[k] - s0[k]; active[k] = 1 unless dedup drops it (d[k] <= W).
 * Any output pointer may be NULL.  Host pointers. */
int fibattn_rung_params(float alpha, const float* offsets, int K, int W, int no_dedup, int round_offsets,
                        float* d, int* s0, float* w, int* active);

/* Base sequences (Section 2): kind 0 = Fibonacci 1,2,3,5,... ; kind 1 =
 * powers of two 1,2,4,... .  Writes K floats to host array f. */
int fibattn_base(int kind, int K, float* f);

/* Per-layer alpha schedules (Section 2, "The per-layer scalar"):
 * kind 0 fixed (alpha = 1); 1 learned (alpha_l = 0.5 + sigmoid(theta[l]));
 * 2 linear stagger (alpha_l = 0.5 + l/(L-1)); 3 coprime reassignment of the
 * linear multiset, layer l takes linear index (stride*l mod L).
 * theta is read only for kind 1.  Host arrays. */
int fibattn_alpha_schedule(int kind, int L, const float* theta, int stride, float* alpha);

/* Inverse of the learned map on [0.5, 1.5]: theta[l] = log((alpha[l] - 0.5) /
 * (1.5 - alpha[l])), the ends (theta = -/+ infinity) clamped to -/+ 30; used to
 * start a learned theta at a static schedule's alpha.  Host arrays. */
int fibattn_theta_of_alpha(int L, const float* alpha, float* theta);

/* ---------------------------------------------------------------------------
 * Coverage of a layer stack (Section 4.2, "Why staggering widens coverage"):
 * the distinct key distances i - j a query reads.  Layer l (alpha = alphas[l])
 * reads D_l = {0..W} plus, for each active rung with d_k <= T-1 (the rung
 * prep of fibattn_rung_params, with T's reach), the floor row's distance
 * floor(d_k) and, when d_k is fractional, the far row's floor(d_k)+1.
 * Outputs (each may be NULL): per_layer[l] = |D_l| (L ints); union_count =
 * |union of D_l|; beyond_window = |union of D_l minus {0..W}|; two_hop =
 * |union over l of {a + b < T : a in D_l, b in D_l+1}| (what a query's
 * representation after two successive layers draws on).  Host arrays;
 * 1 <= L <= 4096, 1 <= T <= 1<<20.
 * ------------------------------------------------------------------------- */
int fibattn_coverage(int L, const float* alphas, const float* offsets, int K, int W, int T, int no_dedup,
                     int* per_layer, int* union_count, int* beyond_window, int* two_hop);

/* ---------------------------------------------------------------------------
 * Shared-memory staging layout of the tensor-core kernels (host-side, no GPU;
 * a diagnostic without counterpart in the paper).  A CTA of these kernels owns
 * a tile of 120 consecutive queries (kind 0: the forward and the backward
 * query pass) or keys (kind 1: the backward key pass) and stages the rows its
 * warps read: for kind 0 the window band [-Wp, 121) and, per staged rung k,
 * the slab [-s0_k - 1, 121 - s0_k) relative to the tile's first query (Wp =
 * 0, 8 or 16 for W = 0, <= 8, <= 16); for kind 1 the band [0, 121 + Wp) and
 * the slabs [s0_k, s0_k + 121) relative to the first key.  Overlapping row
 * ranges are merged and each merged interval is rounded up to whole 8-row
 * copies.  Outputs (host arrays of at least 17 ints, any may be NULL):
 * n_iv intervals with relative first row iv_start, row count iv_len and first
 * shared row iv_smem; slab_row[k] (K ints) = shared row of the first row of
 * rung k's slab, -1 when the rung is not staged (dropped by dedup or beyond
 * T's reach).  FIBATTN_ERR_UNSUPPORTED when the tensor-core kernels do not
 * apply (W > 16 or K > 16).
 * ------------------------------------------------------------------------- */
int fibattn_staging_layout(int kind, int T, int W, float alpha, const float* offsets, int K, int no_dedup,
                           int* n_iv, int* iv_start, int* iv_len, int* iv_smem, int* slab_row);

/* ---------------------------------------------------------------------------
 * Forward without a caller-provided workspace.  The paper has no counterpart;
 * this serves callers that cannot allocate device memory -- a host framework
 * that owns all device memory and gives its plugins only tensors, or a hot
 * path where cudaMalloc's implicit device synchronisation is not allowed.
 * Same arguments and results as fibattn_fwd without workspace/workspace_bytes.
 * Scratch: one library-owned device array of FIBATTN_NOALLOC_SCRATCH_BYTES
 * (32 MiB, enough for B*Hkv*T <= 262144 bf16 rows or 131072 fp32 rows), held
 * by every GPU that loads the library until the process exits.  Calls that
 * need more are rejected with FIBATTN_ERR_INVALID_ARG before any device work.
 * The call allocates nothing (no cudaMalloc / cudaFree).  The first call on
 * each device looks up the array's device address with that device current;
 * make that first call before any stream capture.  Every call shares the one
 * array and leaves its contents behind: calls that overlap on the GPU (other
 * streams, other host threads) race on it and must be serialised by the caller.
 * ------------------------------------------------------------------------- */
#define FIBATTN_NOALLOC_SCRATCH_BYTES (32u << 20)
int fibattn_fwd_noalloc(const void* q, const void* k, const void* v, void* out, float* lse,
                        int B, int H, int T, int D, int W, float alpha, const float* offsets, int K,
                        int dtype, const fibattn_opts* opts, void* stream);

/* ---------------------------------------------------------------------------
 * What follows the layers in a training step (Section 3, "Model and training":
 * a tied embedding over 32768 tokens, gradients clipped to norm 1).
 *
 * Cross entropy of a linear head, in pieces of the vocabulary, logits not kept:
 *   s[n][v] = sum_d x[n][d] w[v][d],  lse[n] = log sum_v exp s[n][v],
 *   loss[n] = lse[n] - s[n][targets[n]],  0 where targets[n] == ignore_index.
 * x [N][D] and w [V][D] in `dtype`, row-major and contiguous; targets [N]
 * 64-bit; loss, lse [N] fp32 (lse is written for ignored rows too).
 * A target outside [0, V) that is not ignore_index is never read through: its
 * loss is NaN, it adds nothing to the gradients, and status bit 2 is set
 * (fibattn_check_status).  Limits: 0 <= N <= 2^24, 1 <= D <= 8192,
 * 1 <= V <= 2^24.  N == 0 launches nothing but the zeroing of dw.
 * Every product is accumulated in fp32; results do not depend on timing.  How many
 * bits its operands keep follows from the sizes, alike in forward and backward:
 *   N <= 2, or N <= 4 and V*D <= 2^22, with D <= 2048: all of them;
 *   other calls of few rows -- N <= 32 in fp32, and in bf16 if V*D <= 2^22, else
 *     N <= 16 if D <= 1024, N <= 8 if not: fp32 operands, and g between the two
 *     products of the gradient, 22 bits (sums of two tf32 values);
 *   all others: fp32 operands and their g 24 bits (sums of three bf16 values).
 *     With bf16 I/O g is rounded to bf16 (relative to the largest |dloss|, so that
 *     equal weights round nothing), as a bf16 tensor between two library calls would
 *     be; it keeps 24 bits in calls of at most 2^26 products, N and V counted up to
 *     multiples of 256.
 * As in any matrix product, an ignored row of x that holds an infinity or NaN
 * still reaches dw as 0 * NaN.
 * ------------------------------------------------------------------------- */
size_t fibattn_linear_xent_fwd_workspace_bytes(int N, int D, int V, int dtype);

int fibattn_linear_xent_fwd(const void* x, const void* w, const long long* targets,
                            float* loss, float* lse,
                            int N, int D, int V, long long ignore_index, int dtype,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Gradient of sum_n dloss[n] * loss[n] (dloss [N] fp32, on the device), with
 * lse from the forward of the same x and w:
 *   g[n][v] = dloss[n] (exp(s[n][v] - lse[n]) - [v == targets[n]]), 0 for ignored rows;
 *   dx = g w [N][D],  dw = g^T x [V][D], in `dtype`, overwritten.
 * The logits are formed again, a piece of the vocabulary at a time; g of one
 * piece is held in the workspace: at most 512 MiB of it, or 256 columns where
 * those are more (512 N bytes in bf16, 1536 N in fp32).  Calls of few rows (the
 * second kind above) hold g of all columns, N rounded up to 8, 16 or 32, in fp32
 * (at most 128 V bytes).  dx or dw may be NULL
 * when only the other is wanted (a frozen head; a probe on frozen states).  They
 * may not alias each other, an input or the workspace. */
size_t fibattn_linear_xent_bwd_workspace_bytes(int N, int D, int V, int dtype);

int fibattn_linear_xent_bwd(const void* x, const void* w, const long long* targets,
                            const float* lse, const float* dloss,
                            void* dx, void* dw,
                            int N, int D, int V, long long ignore_index, int dtype,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Global norm of n tensors and clipping:
 *   norm = sqrt(sum of the squares of all values),
 *   out_i = grad_i * min(1, max_norm / (norm + 1e-6)).
 * grads, outs, numels and dtypes are HOST arrays of n entries, read during the
 * call only; grads[i] and outs[i] are device pointers to numels[i] >= 0
 * contiguous values of dtypes[i], aligned to their element (any view of a flat
 * buffer will do).  outs == NULL: the norm alone.  outs[i] == grads[i] clips
 * in place (and, with norm below max_norm, writes nothing); otherwise an out
 * may not overlap a grad or another out.  max_norm >= 0 (infinity: no
 * clipping).  norm: device, 1 float.  It is not finite if a value is not, or if
 * it is itself beyond fp32; it then passes into the outputs by the formula above
 * (NaN, or 0 with NaN where the infinities were), and the caller that wants to
 * skip such a step looks at norm.  Squares are summed in fp32 in runs of at most
 * 129 values, four runs to a thread are added in fp32, and all beyond in fp64;
 * values whose squares leave fp32's range (above 1.8e19, tiny ones) are squared
 * in fp64.  The result does not depend on timing. */
size_t fibattn_clip_grads_workspace_bytes(int n);

int fibattn_clip_grads(int n, const void* const* grads, void* const* outs,
                       const long long* numels, const int* dtypes, float max_norm,
                       float* norm, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Generating with the attention: a paged cache of keys and values, and the
 * attention of new tokens over it (Section 2, "Attended set": the same window
 * and rungs as fibattn_fwd, of queries that come later than the keys).
 *
 * A cache is two pools of pages for one layer, keys (RoPE-rotated; fp16 for
 * bf16 I/O, fp32 for fp32 I/O, as in fibattn_opts.rotated_k) and values (the I/O
 * type), both [pages][page_rows][Hkv][64] with the same strides, and a table
 * [seqs][pages_per_seq] of 32-bit page numbers on the device.  Storage slot j of
 * sequence b is row j % page_rows of page table[b][j / page_rows].  Strides are
 * in elements, the last dimension is contiguous and the others are any multiples
 * of 64 (a layer of a larger pool, pages with the heads before the rows, ...);
 * the pools start on 32 bytes.
 * Limits: pages_per_seq * page_rows <= 2^30; every row's offset, counted in rows
 * of 64, below 2^32.
 *
 * Tokens lie behind one another, whichever sequence they belong to: token n of
 * N belongs to sequence seqs[n] (seqs NULL: sequence n) and stands at
 * positions[n], both 32-bit on the device, so that a captured call can be replayed
 * for other positions.  A token with a negative position or sequence is padding:
 * fibattn_cache_append writes nothing for it, the attention writes out = 0 and
 * lse = -infinity.
 *
 * What does not exist is never read or written: a sequence that is not in the
 * table, a slot beyond pages_per_seq pages, a page outside the pool (an unused
 * table entry, say -1).  An append then leaves the token out, an attention gives
 * NaN for the token's out and lse, and status bit 3 is set (fibattn_check_status).
 * Pages that no query reads may be taken from a sequence at any time: a query
 * reads no further back than max(W, ceil(largest d_k)).
 *
 * fibattn_cache_init checks a cache's arguments and fills *c with them and with
 * what follows from rope_base (0: 1e4); it touches no device memory.  *c is read
 * by the calls below during the call only, and may be copied.  Its fields are not
 * for the caller to change.
 * ------------------------------------------------------------------------- */
typedef struct {
    void* k_pages;
    void* v_pages;
    const int* table;
    long long page_stride, row_stride, head_stride;
    int pages, page_rows, Hkv, seqs, pages_per_seq, dtype;
    unsigned ready;
    unsigned long long phase[32];
} fibattn_cache;

int fibattn_cache_init(fibattn_cache* c, void* k_pages, void* v_pages, int pages, int page_rows, int Hkv, int D,
                       long long page_stride, long long row_stride, long long head_stride,
                       const int* table, int seqs, int pages_per_seq, int dtype, float rope_base);

/* Writes N tokens' keys, rotated at positions[n], and values into the cache, at
 * storage slot slots[n] (32-bit, on the device; NULL: at slot positions[n]).  k and
 * v: [N][Hkv][64] in the cache's I/O type, contiguous in the last dimension, with
 * strides in elements that are multiples of 16 bytes.  Two tokens of one call at
 * the same slot of the same sequence leave that slot with a mixture of both;
 * nothing else is affected. */
int fibattn_cache_append(const fibattn_cache* c, const void* k, long long k_token_stride, long long k_head_stride,
                         const void* v, long long v_token_stride, long long v_head_stride,
                         const int* positions, const int* slots, const int* seqs, int N, void* stream);

/* Attention of N tokens over the cache: q [N][H][64] as k above (H a multiple of
 * the cache's Hkv; query head h reads head h / (H / Hkv)), out [N][H][64]
 * contiguous and on 16 bytes, lse [N][H] fp32, contiguous.  The query at position p
 * reads slots p .. p-W and, for every active rung with d_k <= p, slots p - floor(d_k)
 * and, where d_k is no integer, p - floor(d_k) - 1: its own key and value too, which
 * have to be appended before.  opts: scale, no_dedup and round_offsets are used; the
 * other fields have to be zero (rope_base is the cache's).  Products and sums are
 * fp32; q is rotated in fp32 and not rounded (bf16: the weights of the values keep 16
 * bits; q keeps 22 bits of what is 2^-29 of its head's largest value or more, and of
 * smaller values all but 2^-50 of that largest).  A value that is not finite gives
 * outputs that are not, of the heads that read it and of no others.  So does a key,
 * but for scores of -infinity, which count for nothing (where there are no others out
 * is NaN and lse -infinity): an infinite key gives those, or NaN, by the signs of q's
 * rotated values that meet it (NaN also for 0, in bf16 for what is below 2^-39 of the
 * head's largest).  Limits of W, K and alpha as for fibattn_fwd; 0 <= N, N * H < 2^31. */
int fibattn_cached_fwd(const fibattn_cache* c, const void* q, long long q_token_stride, long long q_head_stride,
                       void* out, float* lse, const int* positions, const int* seqs, int N, int H, int W,
                       float alpha, const float* offsets, int K, const fibattn_opts* opts, void* stream);

/* The same for drafted tokens that form trees: parents[n] is the token (row of this
 * batch, before n) that token n continues, or -1 if it continues the cached
 * sequence itself; its position is one more than its parent's.  The ancestor at
 * distance j, j steps up (0: the token itself), is read from storage slot
 * slots[ancestor], where fibattn_cache_append put it; what lies further back than
 * the root from the slot of its position.  A parent that is not before its child, and
 * an ancestor that is read but is of another sequence or at another position, count
 * as ones that do not exist (above). */
int fibattn_tree_fwd(const fibattn_cache* c, const void* q, long long q_token_stride, long long q_head_stride,
                     void* out, float* lse, const int* positions, const int* parents, const int* slots,
                     const int* seqs, int N, int H, int W,
                     float alpha, const float* offsets, int K, const fibattn_opts* opts, void* stream);

/* ---------------------------------------------------------------------------
 * Opt-in kernel timing (no counterpart in the paper; used to attribute time
 * to kernels).  fibattn_profile_enable(1) clears the record and brackets every
 * later launch with CUDA events on the launch stream; (0) stops and clears.
 * Launches made while the stream is being captured into a CUDA graph record
 * external event nodes, so the summary then reports the graph's last replay.
 * fibattn_profile_summary(-1, ...) returns the number of distinct kernels
 * recorded; with index i >= 0 it synchronises on those events and writes the
 * kernel name, its summed device time in ms and its launch count.
 * ------------------------------------------------------------------------- */
int fibattn_profile_enable(int on);
int fibattn_profile_summary(int index, char* name, int name_len, double* total_ms, int* launches);

#ifdef __cplusplus
}
#endif

#endif /* FIBATTN_H */
