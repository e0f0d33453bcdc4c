/*
 * meteora.h - C ABI of the MI355X (gfx950) MeteoRA linear-layer forward.
 *
 * The layer (paper Sec. 3.1, Eq. 2 and Eq. 3; row-vector convention of Eq. 1):
 *
 *     G(x) = x * W_gate (+ bias)                      gate logits, fp32
 *     I(x) = top-k adapters by logit (ties -> lower index)
 *     w_i  = softmax over the k selected logits       Eq. 3
 *     o    = x * W_base + scale * sum_{i in I(x)} w_i * ((x * A_i) * B_i)   Eq. 2
 *
 * with the n LoRA pairs stacked contiguously as in Sec. 3.3:
 * A[N, d_in, r], B[N, r, d_out].
 *
 * Conventions common to every entry point
 *  - Every pointer is a DEVICE pointer (HBM of the current HIP device) unless
 *    it is marked "host".  All arrays are dense, row-major, 16-byte aligned.
 *  - `dt` is the storage type of x, W, A, B and out: METEORA_BF16 (bfloat16,
 *    fp32 accumulation) or METEORA_F32.  W_gate, gate_bias, logits and topk_w
 *    are always fp32; indices are int32.
 *  - Storage: x[T, d_in]; W[d_out, d_in] (o[t,c] = sum_i x[t,i] * W[c,i]);
 *    W_gate[d_in, N]; gate_bias[N] or NULL; A[N, d_in, r]; B[N, r, d_out];
 *    out[T, d_out].
 *  - Ownership: the caller owns all memory.  The library never allocates,
 *    frees or keeps device memory; scratch space is the caller's `ws`
 *    (at least meteora_workspace_bytes(...) bytes, 256-byte aligned).
 *    Inputs are only read; outputs are fully overwritten (except
 *    accumulate=1).  Outputs must not alias inputs.
 *  - Execution: all work is enqueued on `stream` (a hipStream_t passed as
 *    void*; NULL = the default stream).  No call synchronises with the host.
 *    Results are deterministic: same inputs -> bit-identical outputs.
 *    Calls that share a workspace must be ordered on one stream.
 *  - Errors: a status code is returned, nothing is thrown.  Arguments are
 *    validated on the host before any launch, so an error status means that
 *    nothing was enqueued.  T == 0 returns METEORA_OK without a launch.
 *  - Limits: 1 <= k <= N <= 64, k <= 8, 1 <= r <= 64; d_in % 8 == 0 and
 *    d_out % 8 == 0; T * k < 2^31.  Inputs must be finite.
 */
#ifndef METEORA_H
#define METEORA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    METEORA_OK = 0,
    METEORA_ERR_INVALID_ARG = 1, /* null required pointer, negative size, k<1, k>N, non-finite scale */
    METEORA_ERR_UNSUPPORTED = 2, /* shape/dtype/alignment outside the limits above */
    METEORA_ERR_WORKSPACE = 3,   /* ws is NULL or ws_bytes too small */
    METEORA_ERR_HIP = 4,         /* a HIP launch reported an error */
    METEORA_ERR_TOO_LARGE = 5    /* beyond the fixed scratch of an entry point that takes no workspace */
} meteora_status;

typedef enum { METEORA_F32 = 0, METEORA_BF16 = 1 } meteora_dtype;

/* A hipStream_t, passed as an opaque pointer so that this header needs no HIP include. */
typedef void* meteora_stream;

/* Library version (major*10000 + minor*100 + patch).  Host only. */
int meteora_version(void);

/* Text for a status code.  Host only; returns a static string. */
const char* meteora_status_string(meteora_status s);

/*
 * Optional set-up of HIP device `device` (-1 = the current device): everything that a kernel's first
 * launch on a device otherwise does by itself, which is one host-side function attribute per kernel
 * that uses more than 64 KB of LDS.  Setting that attribute is not a stream operation and is not
 * allowed while the stream is being captured into a HIP graph: a caller that captures its first call
 * of an entry point runs meteora_init (or one eager call of the same entry point at the same kind of
 * batch size) beforehand.  Cheap to repeat; thread-safe.  Returns METEORA_ERR_HIP without a usable
 * device, METEORA_ERR_INVALID_ARG if `device` cannot be selected.  Leaves the current device unchanged.
 */
meteora_status meteora_init(int device);

/*
 * Scratch bytes needed by meteora_gate_topk, meteora_bucket_tokens,
 * meteora_lora_forward and meteora_linear_forward for this problem size and for
 * any smaller T (the maximum over the four; entry points that take no d_out or
 * r accept the value computed with any legal d_out, r, e.g. 8 and 1).
 * Host only, no HIP call.  Returns 0 for arguments outside the limits.
 */
size_t meteora_workspace_bytes(int T, int d_in, int d_out, int N, int r, int k, meteora_dtype dt);

/*
 * Audit of the workspace carving of meteora_linear_forward (with_packed = 0) or
 * meteora_linear_forward_packed with a blob (with_packed = 1), for tests.  Host only, no HIP call.
 * Entry i of the host arrays (each may be NULL) receives region i's name (static string), its
 * byte offset in ws, the bytes reserved for it, and the bytes that the launch sequence this
 * shape selects writes there (from that sequence's own tile and K-split counts).  Returns the
 * number of regions (at most max_regions entries are filled), or -1 for arguments outside the
 * limits.  Every written extent must fit its reservation, and offset + reserved must stay inside
 * meteora_workspace_bytes.
 */
int meteora_workspace_regions(int T, int d_in, int d_out, int N, int r, int k, meteora_dtype dt,
                              int with_packed, const char** names /*host*/, size_t* offset /*host*/,
                              size_t* reserved /*host*/, size_t* written /*host*/, int max_regions);

/*
 * Gate network and top-k routing (Sec. 3.1: G(x), I(x); Eq. 3).
 *   logits[t,j]  = sum_i x[t,i] * W_gate[i,j] (+ gate_bias[j]), fp32 accumulation
 *   topk_idx[t,:] = the k adapters with the largest logits, listed by descending
 *                   logit, equal logits by ascending adapter index
 *   topk_w[t,:]   = exp(g - g_max) / sum over the k selected (Eq. 3), fp32
 * `logits` ([T,N] fp32) may be NULL if the caller does not want them.
 * inv_temperature scales the selected logits inside the softmax only
 * (1.0f = Eq. 3 as printed; 1/tau for the temperature of App. A.6).
 */
meteora_status meteora_gate_topk(const void* x, const float* W_gate, const float* gate_bias,
                                 int T, int d_in, int N, int k, meteora_dtype dt,
                                 float inv_temperature,
                                 int32_t* topk_idx /*[T,k]*/, float* topk_w /*[T,k]*/,
                                 float* logits /*[T,N] or NULL*/,
                                 void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Token-to-adapter bucketing: the per-adapter token sets {x | i in I(x)} of
 * Sec. 3.3 as index lists instead of gathered copies.
 *   counts[j]  = number of (token, slot) pairs routed to adapter j
 *   offsets    = exclusive prefix sum of counts, offsets[N] = T*k
 *   bucket_tok / bucket_slot [offsets[j] .. offsets[j+1]) = the pairs of adapter
 *                j, ordered by ascending token, then ascending slot (stable)
 * topk_idx values must lie in [0, N).
 */
meteora_status meteora_bucket_tokens(const int32_t* topk_idx /*[T,k]*/, int T, int k, int N,
                                     int32_t* counts /*[N]*/, int32_t* offsets /*[N+1]*/,
                                     int32_t* bucket_tok /*[T*k]*/, int32_t* bucket_slot /*[T*k]*/,
                                     void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * meteora_bucket_tokens for callers that cannot allocate device memory and have no workspace to pass:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same inputs,
 * outputs, order and bit-exact results; the per-chunk histograms that the other entry point keeps in
 * `ws` live in a fixed 256 KiB device array inside the library (one copy per GPU, held until the
 * process ends), so the call allocates nothing and frees nothing.
 *   Limit: T <= 65536 tokens (any k <= 8, N <= 64); beyond that METEORA_ERR_TOO_LARGE, nothing is launched.
 *   The array's device address is looked up on the first call on each device (or by meteora_init).
 *   All calls on one GPU share the array: calls that can overlap on one GPU (different streams with
 *   no ordering between them, or several host threads) race on it and must be serialised by the
 *   caller.  Nothing in it needs clearing between calls: the histogram pass overwrites every entry
 *   the scatter pass reads, so a call may follow a larger one.
 * Other errors as for meteora_bucket_tokens.
 */
meteora_status meteora_bucket_tokens_noalloc(const int32_t* topk_idx /*[T,k]*/, int T, int k, int N,
                                             int32_t* counts /*[N]*/, int32_t* offsets /*[N+1]*/,
                                             int32_t* bucket_tok /*[T*k]*/, int32_t* bucket_slot /*[T*k]*/,
                                             meteora_stream stream);

/*
 * LoRA term of Eq. 2 for a given routing:
 *   delta[t,:] = scale * sum_j topk_w[t,j] * ((x[t,:] * A[a]) * B[a]),  a = topk_idx[t,j]
 *   accumulate = 0: out = delta;  accumulate = 1: out = out + delta.
 * Runs bucketing, the grouped shrink (h = x*A_a, fp32) and the grouped expand.
 */
meteora_status meteora_lora_forward(const void* x, const void* A, const void* B,
                                    const int32_t* topk_idx, const float* topk_w,
                                    int T, int d_in, int d_out, int N, int r, int k,
                                    float scale, meteora_dtype dt,
                                    void* out /*[T,d_out]*/, int accumulate,
                                    void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Whole layer, Eq. 2: out = x*W + scale * sum_{i in I(x)} w_i * ((x*A_i)*B_i),
 * with I(x), w from the gate as in meteora_gate_topk.  inv_temperature as there:
 * 1.0f is Eq. 3 as printed, 1/tau the softmax temperature that App. A.6 uses for the
 * composite tasks (tau = 15, 20, 30); it changes the weights, never the selection.
 * With k = 1 (the top-1 strategy of App. A.1) the weight is exactly 1: no exponential is
 * evaluated, and the per-token work of the shrink and expand is that of one adapter.
 * If topk_idx_out / topk_w_out are not NULL they receive the routing used.
 * Errors: a non-finite scale or inv_temperature is METEORA_ERR_INVALID_ARG.
 */
meteora_status meteora_linear_forward(const void* x, const void* W, const float* W_gate,
                                      const float* gate_bias, const void* A, const void* B,
                                      int T, int d_in, int d_out, int N, int r, int k,
                                      float scale, float inv_temperature, meteora_dtype dt,
                                      void* out /*[T,d_out]*/,
                                      int32_t* topk_idx_out /*[T,k] or NULL*/,
                                      float* topk_w_out /*[T,k] or NULL*/,
                                      void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Weight packing, done once when the adapters are loaded: the stacked adapter
 * tensors of Sec. 3.3 and the gate weight are static during inference, so their
 * kernel-side layouts (W_gate split into three bf16 terms in matrix-core operand
 * order, A in operand order, B transposed, and the gate terms with every column of
 * every A_i as the rows of one matrix for the mid-sized-batch routing kernel) need
 * not be rebuilt for every batch.
 *   meteora_packed_bytes   size of the packed blob for these shapes (0 if this dtype
 *                          uses no packed operands, e.g. METEORA_F32).  Host only.
 *   meteora_pack_weights   fills `packed` (device, 256-byte aligned, caller-owned) from
 *                          W_gate[d_in,N] fp32, A[N,d_in,r], B[N,r,d_out]; enqueued on
 *                          `stream`.  The blob is valid for exactly these tensors and
 *                          shapes; repack after changing any of them.
 *   meteora_linear_forward_packed   meteora_linear_forward that reads the blob instead
 *                          of repacking into the workspace.  `packed` = NULL behaves as
 *                          meteora_linear_forward.  The results are bit-identical.
 *                          W_gate, A and B are still required and must be the tensors the
 *                          blob was packed from: some paths read them directly (fp32 all three;
 *                          decode-sized batches and a few hundred tokens B).
 * Errors: METEORA_ERR_WORKSPACE if packed_bytes is smaller than meteora_packed_bytes.  One smaller size
 * is taken by the forward calls: for d_in % 64 != 0, r % 8 != 0, N > 32 or 3*32 + N*r > 640 the blob once ended in
 * front of its last operand, the matrix of gate terms and adapter columns, (3*NP + N*R) * d_in * 2 bytes
 * (NP = 32 or 64 >= N, R = r rounded up to a multiple of 8).  A blob kept from then, or cut there, gives the same
 * results; a call that reads that matrix packs it into the workspace every time (batches of any other size
 * read what the blob holds), and a group with such a member runs member by member.
 */
size_t meteora_packed_bytes(int d_in, int d_out, int N, int r, meteora_dtype dt);

meteora_status meteora_pack_weights(const float* W_gate, const void* A, const void* B,
                                    int d_in, int d_out, int N, int r, meteora_dtype dt,
                                    void* packed, size_t packed_bytes, meteora_stream stream);

meteora_status meteora_linear_forward_packed(const void* x, const void* W, const float* W_gate,
                                             const float* gate_bias, const void* A, const void* B,
                                             const void* packed, size_t packed_bytes,
                                             int T, int d_in, int d_out, int N, int r, int k,
                                             float scale, float inv_temperature, meteora_dtype dt,
                                             void* out /*[T,d_out]*/,
                                             int32_t* topk_idx_out /*[T,k] or NULL*/,
                                             float* topk_w_out /*[T,k] or NULL*/,
                                             void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Several MeteoRA layers on the same input: the layers of a decoder block that share x (q/k/v, and
 * gate/up; Sec. 4.1 embeds the adapters in all seven linear layers) each have their own base weight,
 * gate and adapters but the same T, d_in, N, r, k, scale and inv_temperature.  The result is that of one
 * meteora_linear_forward_packed call per member (same routing; outputs equal to bf16 accuracy, the
 * split-K sums may run in another order).  For decode-sized batches (T <= 64) and for batches of a few
 * hundred tokens whose members have few output tiles in all (at most 320 tiles of 128 x 128, routing
 * products included), with bf16, packed weights and at most 4 members, the whole group runs in two
 * launches instead of that many per layer; otherwise the members run one after the other.
 *   members  host array of G descriptors; every pointer in it is a device pointer with the meaning and
 *            alignment it has in meteora_linear_forward_packed (packed may be NULL: that member is then
 *            repacked into the workspace on every call, and the group runs member by member).
 *   ws       at least meteora_group_workspace_bytes(d_out[0..G), ...) bytes, 256-byte aligned.
 * Errors as for meteora_linear_forward_packed; G < 1 or G > 64 is METEORA_ERR_INVALID_ARG.
 */
typedef struct {
    const void* W;            /* [d_out, d_in] */
    const float* W_gate;      /* [d_in, N] */
    const float* gate_bias;   /* [N] or NULL */
    const void* A;            /* [N, d_in, r] */
    const void* B;            /* [N, r, d_out] */
    const void* packed;       /* blob of meteora_pack_weights for this member, or NULL */
    size_t packed_bytes;
    int d_out;
    void* out;                /* [T, d_out] */
    int32_t* topk_idx_out;    /* [T,k] or NULL */
    float* topk_w_out;        /* [T,k] or NULL */
} meteora_group_member;

size_t meteora_group_workspace_bytes(const int* d_out /*host, [G]*/, int G, int T, int d_in, int N, int r, int k,
                                     meteora_dtype dt);

meteora_status meteora_linear_forward_group(const void* x, const meteora_group_member* members /*host*/, int G,
                                            int T, int d_in, int N, int r, int k, float scale,
                                            float inv_temperature, meteora_dtype dt,
                                            void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Gradients of the gate of one module for its training (Sec. 3.2, Eq. 4; App. "Top-k strategy"): W, A and B
 * stay fixed, the loss reaches W_gate and gate_bias
 *   - through the output: dy[T,d_out] = dL_lm/do (storage type dt).  With v_j = scale * (x*A_a)*B_a,
 *     a = topk_idx[t,j]:  dL/dw_j = <dy[t], v_j>,  dL/dg_a = w_j * (dL/dw_j - sum_i w_i * dL/dw_i)
 *     (softmax of Eq. 3 over the k selected; the selection itself carries no gradient; zero for k = 1);
 *   - through the LoRA-classification loss of the module, beta * sum_t CE(softmax over all N logits of token
 *     t, labels[t]):  dL/dg_n += beta * (softmax(g)_n - [n == labels[t]]).  labels[t] outside [0, N) gives
 *     token t no classification part; labels == NULL or beta == 0 leaves the term out.
 * Outputs (fp32, overwritten):  d_logits[T,N] (may be NULL),  dW_gate[d_in,N] = x^T * d_logits,
 * dbias[N] = sum_t d_logits[t] (may be NULL).
 * The logits are recomputed from x and the packed weights with the forward call's arithmetic (three-term bf16
 * split of W_gate, fp32 sums over K splits; the number of splits, and with it the last bits, can differ from the
 * forward call's).  topk_idx / topk_w (both or neither): the routing the forward call returned, to be used
 * as it is; NULL ranks again from the recomputed logits (the same routing unless two logits tie to fp32 accuracy).
 * dx[T,d_in] (storage type dt, optional): the gradient with respect to the module's input, for the modules
 * in front of this one:  dx = dy*W + scale * sum_j w_j * ((dy*B_a^T)*A_a^T) + d_logits*W_gate^T  (base projection,
 * selected adapters, gate).  It needs A[N,d_in,r], W_gate[d_in,N] and W_t = the base weight TRANSPOSED, stored
 * [d_in,d_out] (the frozen base weight is kept in both orientations by a caller that trains); with dx == NULL
 * these three may be NULL.  The gate term is computed from two-term bf16 splits (about 2^-16 of its size).
 * `packed` is the blob of meteora_pack_weights for these adapters; B is the stacked [N,r,d_out] tensor.
 * forward_ws (optional): the workspace in which meteora_linear_forward(_packed) ran on this same x, these
 * adapters and the same T, d_in, d_out, N, r, k, dt, not written to since.  For T > 64 (beyond 8192 tokens where
 * the call takes its dense routing products) it leaves its products of x with the packed gate and A operands there and
 * they are read instead of being computed again (one launch less); otherwise the argument is ignored.  The caller vouches
 * for the contents.
 * Limits: dt == METEORA_BF16, N <= 32, r % 8 == 0, d_in % 64 == 0, d_out % 64 == 0, 3*32 + N*r <= 640,
 * T <= 65536; otherwise METEORA_ERR_UNSUPPORTED (meteora_gate_backward_workspace_bytes returns 0).
 * All pointers but the host-side scalars are device memory; ws as for the other entry points.
 */
size_t meteora_gate_backward_workspace_bytes(int T, int d_in, int d_out, int N, int r, int k, meteora_dtype dt);

meteora_status meteora_gate_backward(const void* x /*[T,d_in]*/, const void* dy /*[T,d_out]*/,
                                     const float* gate_bias /*[N] or NULL*/, const void* B /*[N,r,d_out]*/,
                                     const void* packed, size_t packed_bytes,
                                     const int32_t* topk_idx /*[T,k] or NULL*/, const float* topk_w /*[T,k] or NULL*/,
                                     const int32_t* labels /*[T] or NULL*/, float beta,
                                     int T, int d_in, int d_out, int N, int r, int k, float scale, meteora_dtype dt,
                                     float* dW_gate /*[d_in,N]*/, float* dbias /*[N] or NULL*/,
                                     float* d_logits /*[T,N] or NULL*/,
                                     const void* A /*[N,d_in,r] or NULL*/, const float* W_gate /*[d_in,N] or NULL*/,
                                     const void* W_t /*[d_in,d_out] or NULL*/, void* dx /*[T,d_in] or NULL*/,
                                     const void* forward_ws /*or NULL*/, size_t forward_ws_bytes,
                                     void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * The paper's own schedules of Eq. 2 (Sec. 3.3), as baselines to measure against on the same GPU.  Same
 * arguments, result and routing as meteora_linear_forward (inv_temperature = 1); only the LoRA term is
 * scheduled differently, from this library's gate, bucketing and GEMM kernels plus plain gather / scatter /
 * batched-product kernels.  Not part of the layer's own path.
 *   METEORA_VARIANT_LOOP_ORIGINAL  "loop-original": for each adapter i in turn, gather the tokens routed to it
 *       (X_i), two GEMMs (X_i A_i) B_i, weighted scatter-add into out.  The launch shapes depend on the
 *       routing, so the call SYNCHRONISES `stream` once to read the per-adapter counts on the host (it cannot
 *       be captured into a HIP graph); up to 4 launches per non-empty adapter.
 *   METEORA_VARIANT_BMM_GATHER     Eq. 5 ("bmm-torch"): A_{I(t)_j} and B_{I(t)_j} are copied for every
 *       (token, slot) pair (T*k/N times the size of the stacked adapters, the cost Sec. 3.3 names), then two
 *       batched products over the T*k pairs and the weighted sum over the k slots.
 * Intermediates are stored in dt (X_i A_i, (X_i A_i) B_i and the running output are rounded to bf16 for
 * METEORA_BF16, as a framework-level implementation does), so outputs agree with the layer call to a few
 * bf16 roundings, not bit for bit.
 * Limits: as meteora_linear_forward, and r % 8 == 0.  ws: meteora_variant_workspace_bytes (bmm-gather:
 * about T*k*r*(d_in+d_out) elements).  Errors as for meteora_linear_forward.
 */
typedef enum { METEORA_VARIANT_LOOP_ORIGINAL = 0, METEORA_VARIANT_BMM_GATHER = 1 } meteora_variant;

size_t meteora_variant_workspace_bytes(meteora_variant variant, int T, int d_in, int d_out, int N, int r, int k,
                                       meteora_dtype dt);

meteora_status meteora_variant_forward(meteora_variant variant, const void* x, const void* W, const float* W_gate,
                                       const float* gate_bias, const void* A, const void* B,
                                       int T, int d_in, int d_out, int N, int r, int k, float scale, meteora_dtype dt,
                                       void* out /*[T,d_out]*/, int32_t* topk_idx_out /*[T,k] or NULL*/,
                                       float* topk_w_out /*[T,k] or NULL*/,
                                       void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Base projection alone, first term of Eq. 1 / Eq. 2: out = x * W
 * (W stored [d_out, d_in]).  Exposed so the dense contraction can be checked
 * and timed on its own.
 */
meteora_status meteora_base_gemm(const void* x, const void* W, int T, int d_in, int d_out,
                                 meteora_dtype dt, void* out /*[T,d_out]*/, meteora_stream stream);

/*
 * Rows as 8-bit whole numbers with one scale each: the tokens of an activation, or the output channels of a weight
 * W[d_out, d_in] (its rows).  With a = max_i |x[t,i]|:
 *   scale[t] = a / 127,   q[t,i] = 127 * x[t,i] / a  rounded to the nearest whole number, halves to the even one
 * (the rounding of the exact quotient).  A row of zeros gives zeros and scale 0.  q lies in [-127, 127].  A row that holds an
 * infinity or a NaN gives zeros and scale infinity or NaN, so that its products are NaN and all others what they are.
 * Limits: d % 8 == 0, rows < 2^24.  x in dt; q, scale 16-byte aligned.
 */
meteora_status meteora_quantize_rows(const void* x /*[rows,d]*/, int rows, int d, meteora_dtype dt,
                                     int8_t* q /*[rows,d]*/, float* scale /*[rows]*/, meteora_stream stream);

/*
 * Product of 8-bit whole numbers with a scale per token and per output channel, over groups of consecutive rows:
 *   out[t,c] = q_scale[t] * w_scale[e,c] * sum_i q[t,i] * W[e,c,i],   e = the group with offsets[e] <= t < offsets[e+1]
 * The sum is exact (whole numbers); fp32 scaling, by q_scale first, one rounding where dt (the type of out) is METEORA_BF16.
 *   offsets == NULL: N = 1, all rows are one group: a base projection (the 8-bit counterpart of meteora_base_gemm on rows
 *                    that are quantised already).
 *   offsets[N+1] (device): groups as meteora_sort_tokens and meteora_bucket_tokens return them, one matrix per adapter;
 *                    groups may be empty.  Rows outside every group (t >= offsets[N]) are left as they were in out.
 *                    Offsets must lie in [0, T] and not fall; whatever they hold, only rows in [0, T) are read and written.
 * Integer weights are frozen: there is no gradient for W.  The gradient with respect to the rows that were quantised (the rounding passed
 * by) is dx[t,i] = sum_c dy[t,c] * w_scale[e,c] * W[e,c,i], whose scales lie along the sum: no call of this entry point computes it.  In
 * bf16 it is meteora_base_gemm of a group's dy on the matrix V[i,c] = w_scale[e,c] * W[e,c,i].  In 8 bits it is approximated by this entry point on
 * dy and V quantised anew, each with a rounding of its own: with a = max_c |dy[t,c]| and b = max_c |V[i,c]| off by up to
 *   sum_c (|V[i,c]| * a + |dy[t,c]| * b + a * b / 254) / 254
 * before the roundings of fp32 and of the output.
 * Limits: d_in % 16 == 0, d_in <= 131056, d_out % 8 == 0, d_out <= 2^20, N <= 64, T < 2^24, T * d_out < 2^33.
 */
meteora_status meteora_gemm_i8(const int8_t* q /*[T,d_in]*/, const float* q_scale /*[T]*/, const int8_t* W /*[N,d_out,d_in]*/,
                               const float* w_scale /*[N,d_out]*/, const int32_t* offsets /*[N+1] or NULL*/, int T, int d_in,
                               int d_out, int N, meteora_dtype dt, void* out /*[T,d_out]*/, meteora_stream stream);

/*
 * The kernel that meteora_gemm_i8 starts for these sizes, for tests that mean to reach every one.  Host only, no HIP call.  grouped:
 * offsets are given.  The host pointers (each may be NULL) receive its name (a static string: "one" for up to 128 inputs, "wave" for few
 * rows, "ring" for many), the rows and columns of its tiles, the workgroups that share a CU, whether the weights of a group with a
 * single row tile are requested as read once, and whether a second launch may take the tiles of a last, nearly empty round.  Returns 0, or -1
 * for arguments outside the limits of meteora_gemm_i8 and for T == 0.
 */
int meteora_gemm_i8_kernel(int T, int d_in, int d_out, int N, int grouped, const char** name /*host*/, int* tile_rows /*host*/,
                           int* tile_cols /*host*/, int* per_cu /*host*/, int* read_once /*host*/, int* tail /*host*/);

/*
 * Base projection with the weight in 8 bits: meteora_quantize_rows of x, then meteora_gemm_i8 with one group.  x and out in dt.
 * ws: meteora_base_gemm_i8_workspace_bytes(T, d_in) bytes (the quantised rows and their scales), which also holds any smaller T;
 * 0 for arguments outside the limits of meteora_gemm_i8.
 */
size_t meteora_base_gemm_i8_workspace_bytes(int T, int d_in);

meteora_status meteora_base_gemm_i8(const void* x /*[T,d_in]*/, const int8_t* W /*[d_out,d_in]*/, const float* w_scale /*[d_out]*/,
                                    int T, int d_in, int d_out, meteora_dtype dt, void* out /*[T,d_out]*/, void* ws,
                                    size_t ws_bytes, meteora_stream stream);

/*
 * Rows as 4-bit values with a power of two for every 32 consecutive inputs (a block): the tokens of an activation, or the output
 * channels of a weight W[d_out, d_in].  A code c stands for (-1)^(c >> 3) times 0, 0.5, 1, 1.5, 2, 3, 4, 6 (by c & 7; E2M1), a scale byte E
 * for 2^(E - 127), 255 for NaN (E8M0).  With a = max |x[t,i]| over a block:
 *   E = max(0, floor(log2 a) - 2 + 127),   q[t,i] = the value nearest to x[t,i] * 2^(127 - E), ties to the even code, at most 6,
 * the sign kept.  A block of zeros has E = 0.  A block that holds an infinity or a NaN is zeros with E = 255: products of its row are NaN,
 * all others what they are.
 *   q[rows, d/2]   input 2j of a row in the low, 2j + 1 in the high half of byte j
 *   scale          meteora_mx4_scale_bytes(rows, d) = ceil(d/512) * rows * 16 bytes: block b of row t has its byte at
 *                  [b / 16][t][(b % 4) * 4 + b % 16 / 4]; bytes of no block are zeros (quantising writes them; the products count on it)
 * meteora_dequantize_mx4 gives the values back, out[rows, d], or out[d, rows] with transpose (rows % 8 == 0 then).  They are exact in
 * fp32 and bf16 but for those of 2^128 and more, which are infinite, and in bf16 those below 2^-133, of which there are none in a
 * block that was quantised.
 * Limits: d % 32 == 0, d <= 131072, rows < 2^24, rows * d < 2^36 (0 from meteora_mx4_scale_bytes outside).  x, out in dt.
 */
size_t meteora_mx4_scale_bytes(int rows, int d);

meteora_status meteora_quantize_mx4(const void* x /*[rows,d]*/, int rows, int d, meteora_dtype dt, uint8_t* q /*[rows,d/2]*/,
                                    uint8_t* scale, meteora_stream stream);

meteora_status meteora_dequantize_mx4(const uint8_t* q /*[rows,d/2]*/, const uint8_t* scale, int rows, int d, meteora_dtype dt,
                                      int transpose, void* out /*[rows,d] or [d,rows]*/, meteora_stream stream);

/*
 * Product of such rows and such weights, over groups of consecutive rows:
 *   out[t,c] = sum_i V(q[t,i]) * V(W[e,c,i]),   e = the group with offsets[e] <= t < offsets[e+1],   V: the values stood for
 * Products of two values are exact, sums fp32 in an order that depends on the sizes, one rounding where dt (the type of out) is
 * METEORA_BF16.  offsets, N, groups and rows of no group as in meteora_gemm_i8.  w_scale: the N matrices' scales one behind the other, each
 * meteora_mx4_scale_bytes(d_out, d_in); q_scale: meteora_mx4_scale_bytes(T, d_in).
 * Weights are frozen: there is no gradient for W.  The gradient with respect to the rows that were quantised (the rounding passed by) is
 * dx[t,i] = sum_c dy[t,c] * V(W[e,c,i]): of one matrix meteora_base_gemm_mx4_backward, of groups that entry point once for every group with rows, on
 * the group's rows of dy and its matrix, which takes the offsets on the host; no call computes it for all groups at once.
 * Limits: those of the rows for both operands, d_out % 8 == 0, d_out <= 2^20, N <= 64, T * d_out < 2^33.
 *
 * meteora_gemm_mx4_kernel: the kernel that these sizes lead to, as meteora_gemm_i8_kernel ("one" for up to 256 inputs).
 */
meteora_status meteora_gemm_mx4(const uint8_t* q /*[T,d_in/2]*/, const uint8_t* q_scale, const uint8_t* W /*[N,d_out,d_in/2]*/,
                                const uint8_t* w_scale, const int32_t* offsets /*[N+1] or NULL*/, int T, int d_in, int d_out, int N,
                                meteora_dtype dt, void* out /*[T,d_out]*/, meteora_stream stream);

int meteora_gemm_mx4_kernel(int T, int d_in, int d_out, int N, int grouped, const char** name /*host*/, int* tile_rows /*host*/,
                            int* tile_cols /*host*/, int* per_cu /*host*/, int* read_once /*host*/, int* tail /*host*/);

/*
 * Base projection with the weight in 4 bits: meteora_quantize_mx4 of x, then meteora_gemm_mx4 with one group.  x and out in dt.
 * ws: meteora_base_gemm_mx4_workspace_bytes(T, d_in) bytes, which also holds any smaller T; 0 outside the limits.
 *
 * meteora_base_gemm_mx4_backward: its gradient with respect to x, the rounding of x passed by (the weight is frozen and has none):
 *   dx[t,i] = sum_c dy[t,c] * V(W[c,i])
 * dy and dx in dt, dy as it is (not quantised), fp32 sums, one rounding.  ws holds sums of parts, or beyond some sizes the weight's values,
 * transposed, of every call anew: meteora_base_gemm_mx4_backward_workspace_bytes(d_in, d_out, dt), whatever T (bf16: two bytes a value and more;
 * fp32: four, 32 MB at most for more than 192 outputs).
 */
size_t meteora_base_gemm_mx4_workspace_bytes(int T, int d_in);

meteora_status meteora_base_gemm_mx4(const void* x /*[T,d_in]*/, const uint8_t* W /*[d_out,d_in/2]*/, const uint8_t* w_scale, int T, int d_in,
                                     int d_out, meteora_dtype dt, void* out /*[T,d_out]*/, void* ws, size_t ws_bytes, meteora_stream stream);

size_t meteora_base_gemm_mx4_backward_workspace_bytes(int d_in, int d_out, meteora_dtype dt);

meteora_status meteora_base_gemm_mx4_backward(const void* dy /*[T,d_out]*/, const uint8_t* W /*[d_out,d_in/2]*/, const uint8_t* w_scale, int T,
                                              int d_in, int d_out, meteora_dtype dt, void* dx /*[T,d_in]*/, void* ws, size_t ws_bytes,
                                              meteora_stream stream);

/*
 * Rows next to each other by adapter (the X_i of Sec. 3.3 as rows that are moved; meteora_bucket_tokens lists them):
 *   pos[t,j]   the place of pair (t, j) among all pairs whose topk_idx lies in [0, N), by adapter, then token, then slot;
 *              -1 for other ids (padding tokens, say with -1), which go nowhere
 *   offsets    the first place of every adapter; offsets[N] = the number of places taken, at most T*k.  With T == 0 nothing is
 *              launched and offsets are not written either (the caller clears them where something reads them)
 *   xs         row pos[t,j] is x[t].  Rows from offsets[N] on are left as they were.
 *   xs_scale == NULL: xs[T*k, d] in dt.  Otherwise xs is int8_t[T*k, d], quantised as in meteora_quantize_rows, and xs_scale[T*k]
 *              holds the rows' scales: the operand of meteora_gemm_i8.
 * The gradient with respect to x is meteora_unsort_tokens with w = NULL on the gradient of xs (xs in dt; none through the
 * rounding to 8 bits).
 * Limits: d % 8 == 0, k <= 8 (k may exceed N, and an id may stand twice in a token's row), N <= 64, T < 2^24.
 * ws: meteora_sort_workspace_bytes(T, k, N) bytes, which also holds any smaller T; 0 outside the limits.
 */
size_t meteora_sort_workspace_bytes(int T, int k, int N);

meteora_status meteora_sort_tokens(const void* x /*[T,d]*/, const int32_t* topk_idx /*[T,k]*/, int T, int k, int N, int d,
                                   meteora_dtype dt, void* xs /*[T*k,d]*/, float* xs_scale /*[T*k] or NULL*/,
                                   int32_t* pos /*[T,k]*/, int32_t* offsets /*[N+1]*/, void* ws, size_t ws_bytes,
                                   meteora_stream stream);

/*
 * Back to the order of the tokens, with weights:
 *   out[t] = base[t] + scale * sum_j w[t,j] * ys[pos[t,j]]
 * over the slots whose place lies in [0, rows), rows being those of ys; the others give nothing, and a token without any is
 * base[t], or zeros.  fp32 sums in order of the slots, one rounding.  base == NULL: zeros; base may be out itself.  w == NULL: ones.
 *
 * meteora_unsort_backward, for dy = dL/d out:
 *   dys[pos[t,j]] = scale * w[t,j] * dy[t],    dw[t,j] = scale * <dy[t], ys[pos[t,j]]>   (fp32; 0 where the place is none)
 * Rows of dys that no pos names are left as they were.  dw may be NULL, and then ys too.  The gradient of base is dy.
 * Every place must be named at most once (as meteora_sort_tokens returns them).
 * ys, base, out, dy, dys in dt.  Limits: d % 8 == 0, k <= 8, T < 2^24, rows < 2^31.
 */
meteora_status meteora_unsort_tokens(const void* ys /*[rows,d]*/, int64_t rows, const int32_t* pos /*[T,k]*/,
                                     const float* w /*[T,k] or NULL*/, int T, int k, int d, float scale, meteora_dtype dt,
                                     const void* base /*[T,d] or NULL*/, void* out /*[T,d]*/, meteora_stream stream);

meteora_status meteora_unsort_backward(const void* dy /*[T,d]*/, const void* ys /*[rows,d] or NULL*/, int64_t rows,
                                       const int32_t* pos /*[T,k]*/, const float* w /*[T,k] or NULL*/, int T, int k, int d,
                                       float scale, meteora_dtype dt, void* dys /*[rows,d]*/, float* dw /*[T,k] or NULL*/,
                                       meteora_stream stream);

/*
 * Gated MLPs of experts for a few tokens (T <= 64: a decode step, drafted tokens), routing given:
 *   h[t,j] = silu(W1[e, 0:f] x[t]) * (W1[e, f:2f] x[t]),   e = topk_idx[t,j],   silu(g) = g / (1 + exp(-g))
 *   out[t] = base[t] + scale * sum_j topk_w[t,j] * (W2[e] h[t,j])
 * Ids outside [0, N) (padding tokens, say with -1) give nothing: such a token is base[t], or zeros.  An id may stand twice in a token's
 * row.  base == NULL: zeros; base may be out itself.  x, base, out in dt, which must be METEORA_BF16.  Weights:
 *   w1_scale == w2_scale == NULL:  W1[N,2f,d] and W2[N,d,f] in dt
 *   otherwise                      in 4 bits as meteora_quantize_mx4 gives them, a matrix behind the other: W1 [N,2f,d/2] with N times
 *                                  meteora_mx4_scale_bytes(2f, d), W2 [N,d,f/2] with N times meteora_mx4_scale_bytes(d, f).  Their values
 *                                  enter the products as bf16, exactly; x is not quantised.
 * fp32 sums; h is rounded to bf16, as the operand of the second product, and out once.  The weights of the experts in use are read once (where
 * more than 16 or 32 tokens share an expert, again from the caches).  Without tokens nothing is launched.
 * Limits: T <= 64, N <= 64, k <= 8, d % 8 == 0, f % 8 == 0 (in 4 bits % 32), d, f <= 131072.
 * ws: meteora_experts_workspace_bytes(T, d, f, N, k) bytes, which also holds any smaller T; 0 outside the limits.
 *
 * meteora_moe_forward: the same behind its gate, as meteora_gate_topk routes (k <= N).  The logits' sums are in an order of their own, for one token in
 * another than for more, so that two that are equal to fp32 accuracy may rank the other way there, or in a batch of another size; logits that are equal
 * throughout (columns of W_gate and biases that are equal) go to the lowest index always.  topk_idx_out / topk_w_out receive the routing if they are not NULL.
 * These two have no gradients.
 */
size_t meteora_experts_workspace_bytes(int T, int d, int f, int N, int k);

meteora_status meteora_experts_forward(const void* x /*[T,d]*/, const int32_t* topk_idx /*[T,k]*/, const float* topk_w /*[T,k]*/,
                                       const void* W1, const uint8_t* w1_scale /*or NULL*/, const void* W2,
                                       const uint8_t* w2_scale /*or NULL*/, int T, int d, int f, int N, int k, float scale, meteora_dtype dt,
                                       const void* base /*[T,d] or NULL*/, void* out /*[T,d]*/, void* ws, size_t ws_bytes,
                                       meteora_stream stream);

meteora_status meteora_moe_forward(const void* x /*[T,d]*/, const float* W_gate /*[d,N]*/, const float* gate_bias /*[N] or NULL*/,
                                   const void* W1, const uint8_t* w1_scale /*or NULL*/, const void* W2, const uint8_t* w2_scale /*or NULL*/,
                                   int T, int d, int f, int N, int k, float scale, float inv_temperature, meteora_dtype dt,
                                   const void* base /*[T,d] or NULL*/, void* out /*[T,d]*/, int32_t* topk_idx_out /*[T,k] or NULL*/,
                                   float* topk_w_out /*[T,k] or NULL*/, void* ws, size_t ws_bytes, meteora_stream stream);

/*
 * Optional per-stage timing, for benchmarks.  Host only; off by default.
 * While enabled, meteora_lora_forward and meteora_linear_forward record
 * hipEvents on `stream` around each stage (prep, gate_logits, gate_topk,
 * bucket, shrink, gemm, expand) for up to 256 calls.  A stage's reading is its kernels' time
 * plus the dispatch gap in front of them (about 2 us per launch against a kernel trace).  A stage that a batch size
 * folds into another is not reported: where the routing runs without bucket lists (bf16, T > 64) gate_logits covers
 * the gate logits and the shrink, gate_topk the top-k, softmax and selection (batches with few output tiles:
 * gemm covers the K-split projection with those products, shrink the launch after it); for
 * T <= 64 gemm covers the base projection's split-K launch (with the gate logits and every adapter's shrink),
 * shrink the launch after it (top-k, softmax, reduction, expand); for METEORA_F32 meteora_linear_forward reports gemm
 * (the base projection) and expand (everything after it).  meteora_stage_timing_read waits
 * for those events, returns per stage the summed milliseconds and the number
 * of timed launches (arrays of meteora_stage_count() entries, host memory)
 * and the number of calls covered, and starts a new window.  Not thread-safe;
 * enable/disable must not race with other calls.
 */
int meteora_stage_count(void);
const char* meteora_stage_name(int stage);
meteora_status meteora_stage_timing_enable(int on);
meteora_status meteora_stage_timing_read(float* ms_sum /*host*/, int* launches /*host*/, int* calls /*host*/);

#ifdef __cplusplus
}
#endif
#endif /* METEORA_H */
