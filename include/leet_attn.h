/*
 * leet_attn.h -- C ABI of the MI355X (gfx950) library for exponentially decaying
 * causal linear attention.
 *
 * Operator (Section 2.2, Eq. "BCMV", with B = Q and C = K):
 *
 *     O = ((Q K^T) .* M) V,      M[i][j] = gamma^(i-j) if i >= j, else 0,
 *
 * one gamma per head, 0 <= gamma <= 1, 0^0 = 1 (so M[i][i] = 1 always).  There is
 * no softmax, no row normalisation and no 1/sqrt(d) factor inside the operator.
 * The library evaluates it in chunked ("block-based") form -- Appendix B.2, Alg. 2,
 * carried over to the decaying mask with the row/column weight split of
 * Appendix B.3, Alg. 4 -- and continues it token by token with the row-based
 * recursion of Appendix B.1, Alg. 1 and the discounted update of Appendix C.1:
 *
 *     S <- gamma S + k^T v ;   o = q S            (S is d x d, rows = key index).
 *
 * Conventions shared by every entry point
 *   - Every tensor pointer is a DEVICE pointer (HIP global memory on the current
 *     device), 16-byte aligned, densely packed, row-major in the stated shape.
 *   - `stream` is a hipStream_t passed as void*; NULL means the default stream.
 *     Calls are asynchronous: they enqueue kernels on `stream` and return.  The
 *     caller keeps every buffer alive and unmodified until the stream has
 *     finished the work.
 *   - The caller owns all buffers.  The library keeps no pointer after the work
 *     is done.  `out` must not overlap any input.
 *   - The return value is a leet_status.  Arguments are validated on the host
 *     before anything is enqueued: on every status but LEET_OK and
 *     LEET_ERR_LAUNCH no buffer has been written.  LEET_ERR_LAUNCH means the HIP
 *     runtime failed part-way; the contents of the output buffers are then undefined.
 *   - d must be 64 or 128 (the _rd entry points also take rank 128 with value width
 *     256).  B, H >= 1.  N need not be a multiple of the chunk length (64
 *     tokens); the last chunk may be ragged.
 *   - A prefill over no tokens is legal (N = 0; N < 0 is LEET_ERR_INVALID_ARG): the loop over
 *     chunks (Alg. 2) does not run, so nothing is written to `out`, and `state_out`, when
 *     given, receives the entering state unchanged (zero if `state_in` is NULL).  q, k, v and
 *     out are then empty and may be NULL.  It needs no workspace; the plan query reports zero
 *     segments.  The decode step has no length and always processes one token.
 *   - Outputs that the library will not read again (prefill `out`) are written
 *     with nontemporal stores, so that they do not displace the inputs from the
 *     caches; this changes no value.
 *   - gamma outside [0, 1] is not diagnosed (the values live in device memory).
 */
#ifndef LEET_ATTN_H
#define LEET_ATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LEET_F32 = 0,  /* q, k, v are IEEE binary32; products are those of fp32 over its whole
                      range, on fp32 MFMA (d = 64) or as sums of bf16 MFMA products of
                      three terms an operand (d = 128; segments with values outside the
                      terms' range run on fp32 MFMA, which takes them longer)          */
    LEET_BF16 = 1, /* q, k, v are bfloat16; products on bf16 MFMA, fp32 accumulate  */
    LEET_F16 = 2   /* q, k, v are IEEE binary16; products on fp16 MFMA, fp32 accumulate
                      (accepted by the _v2, _rd and _recurrent entry points)       */
} leet_dtype;

/*
 * Which mask M the operator uses (Section 2.2: the decaying mask of Eq. "BCMV", or the 0/1
 * causal mask of plain causal linear attention, which is the same operator with gamma = 1).
 */
typedef enum {
    LEET_MASK_DECAY = 0, /* M[i][j] = gamma_h^(i-j), i >= j; `gamma` is read                  */
    LEET_MASK_CAUSAL = 1 /* M[i][j] = 1, i >= j; `gamma` is ignored and may be NULL; kernels
                            specialised to skip every decay multiplication                 */
} leet_mask;

typedef enum {
    LEET_OK = 0,
    LEET_ERR_INVALID_ARG = 1, /* NULL required pointer, non-positive size, misaligned pointer, workspace too small */
    LEET_ERR_UNSUPPORTED = 2, /* d not in {64, 128}, unknown dtype or dtype combination, no gfx950 device */
    LEET_ERR_LAUNCH = 3,      /* the HIP runtime refused a launch or an allocation */
    LEET_ERR_TOO_LARGE = 4,   /* sizes overflow the library's index range */
    LEET_ERR_CAPTURE = 5,     /* `stream` is capturing and the library-owned workspace would have to be
                                 allocated or grown; nothing was enqueued */
    LEET_ERR_SCRATCH_LIMIT = 6 /* leet_attn_forward_static: the call's segment states exceed the static
                                 scratch; nothing was enqueued */
} leet_status;

/*
 * Chunked prefill (Eq. "BCMV" via Alg. 2 + the Alg. 4 weight split), zero initial state.
 *   q, k, v  [B][H][N][d], element type `dtype`
 *   gamma    [H] float
 *   out      [B][H][N][d] float (fp32 for both input types)
 * Long sequences are cut into segments that run in parallel; the segment
 * boundary states live in a per-device workspace that the library allocates
 * with hipMalloc on first need.  When a later call needs more, a larger block
 * is allocated and the old one is kept (work in flight or a captured graph may
 * still use it) until leet_attn_release_workspace.  Because that workspace is
 * shared, calls on one device must not run concurrently on different streams;
 * use leet_attn_forward_ex with caller-owned workspaces for that.
 * Under stream capture the library never allocates: if the workspace it owns
 * is too small for the call the status is LEET_ERR_CAPTURE and nothing is
 * recorded.  Make one eager call of the same shape before capturing (the graph
 * then holds an address that stays valid until leet_attn_release_workspace), or
 * capture leet_attn_forward_ex with a caller-owned workspace.
 */
int leet_attn_forward(const void *q, const void *k, const void *v, const float *gamma, float *out,
                      int B, int H, int N, int d, int dtype, void *stream);

/*
 * One decode step (Alg. 1 with the discounted update of Appendix C.1):
 *     S <- gamma_h S + k^T v ;  o = q S     for each (b, h).
 *   q, k, v      [B][H][d] bfloat16
 *   gamma        [H] float
 *   state_inout  [B][H][d][d] float, rows = key index, cols = value index; updated in place
 *   out          [B][H][d] float
 */
int leet_attn_decode_step(const void *q, const void *k, const void *v, const float *gamma,
                          float *state_inout, float *out, int B, int H, int d, void *stream);

/* As leet_attn_decode_step, with q, k, v of element type `dtype` (LEET_F32 or LEET_BF16). */
int leet_attn_decode_step_ex(const void *q, const void *k, const void *v, const float *gamma,
                             float *state_inout, float *out, int B, int H, int d, int dtype,
                             void *stream);

/*
 * Chunked prefill with state hand-off (the state that Alg. 1 carries from token to token,
 * entering and leaving the call), so that a prompt can be processed in pieces and
 * continued by decode steps.
 *   state_in   [B][H][d][d] float or NULL (zero state); the state before token 0
 *   state_out  [B][H][d][d] float or NULL; receives the state after token N-1.
 *              May alias state_in (when the sequences are cut into segments the kernels read
 *              the entering state from a copy in the workspace, so the order in which the
 *              segments run does not matter).
 *   workspace  device buffer of at least leet_attn_workspace_bytes(B, H, N, d, dtype)
 *              bytes, 256-byte aligned, or NULL to use the library's own per-device
 *              workspace as leet_attn_forward does.  Its contents are scratch.
 *   workspace_bytes  size of `workspace` (ignored when workspace is NULL)
 *   segments   0 = let the library choose how many parallel segments to cut each
 *              sequence into; > 0 = request that many (clamped to the number of
 *              chunks).  The result does not depend on it beyond rounding.
 */
int leet_attn_forward_ex(const void *q, const void *k, const void *v, const float *gamma, float *out,
                         const float *state_in, float *state_out,
                         void *workspace, size_t workspace_bytes, int segments,
                         int B, int H, int N, int d, int dtype, void *stream);

/*
 * Chunked prefill with every option: as leet_attn_forward_ex, and additionally
 *   in_dtype   LEET_F32, LEET_BF16 or LEET_F16 (the paper's methods take fp16 and fp32 inputs,
 *              Section 4; bf16 is this library's headline type)
 *   out_dtype  LEET_F32, or, for 16-bit inputs, the input type: `out` is then [B][H][N][d] of
 *              that type, rounded to nearest even from the fp32 accumulators (halves the
 *              output traffic of an HBM-bound kernel)
 *   mask       a leet_mask
 * Any other combination returns LEET_ERR_UNSUPPORTED.  States stay fp32.
 */
int leet_attn_forward_v2(const void *q, const void *k, const void *v, const float *gamma, void *out,
                         const float *state_in, float *state_out,
                         void *workspace, size_t workspace_bytes, int segments,
                         int B, int H, int N, int d, int in_dtype, int out_dtype, int mask, void *stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph capture that has not made
 * an eager call first, tight serving loops, harnesses that forbid hipMalloc): leet_attn_forward_ex
 * with the segment states in a fixed scratch array that is part of the library's device image
 * (leet_attn_static_scratch_bytes() = 32 MiB, held by every GPU that loads the library until the
 * process ends).  The call allocates and frees nothing; q, k, v, gamma, out and the states are
 * the caller's as everywhere else.  Same kernels and same plan as leet_attn_forward_ex, hence
 * bit-identical results.
 *   segments   as for leet_attn_forward_ex.  If the plan's segment states need more than the
 *              scratch holds (leet_attn_workspace_bytes tells), the status is
 *              LEET_ERR_SCRATCH_LIMIT and nothing is enqueued; ask for fewer segments (one
 *              segment needs no scratch at all) or use leet_attn_forward_ex.
 *   dtype      LEET_F32 or LEET_BF16; fp32 output; decaying mask.
 * All calls on one GPU share that GPU's scratch, which keeps the previous call's contents
 * (nothing in it needs clearing: every slot a call reads is first written by that call's own
 * kernels).  Calls that overlap on one GPU -- different streams, or a graph replay beside an
 * eager call -- race on it; serialise them.
 */
int leet_attn_forward_static(const void *q, const void *k, const void *v, const float *gamma, float *out,
                             const float *state_in, float *state_out, int segments,
                             int B, int H, int N, int d, int dtype, void *stream);
size_t leet_attn_static_scratch_bytes(void);

/*
 * Row-based prefill: the same operator evaluated token by token as Alg. 1 (Appendix B.1) states
 * it, with the discounted update of Appendix C.1 -- the decode step iterated over N with the
 * state kept on chip.  No MFMA, sequential in N, parallel over (batch, head) and value columns
 * only.  It is the in-library comparison point for the chunked kernels (the paper's fastest
 * method at batch 16 is of this kind, Section 5.1); the chunked entry points are the fast path.
 *   q, k, v    [B][H][N][d] of `dtype` (LEET_F32, LEET_BF16 or LEET_F16)
 *   out        [B][H][N][d] float
 *   state_in   [B][H][d][d] float or NULL;  state_out  [B][H][d][d] float or NULL (may alias)
 *   mask       a leet_mask (gamma may be NULL for LEET_MASK_CAUSAL)
 * Needs no workspace.
 */
int leet_attn_forward_recurrent(const void *q, const void *k, const void *v, const float *gamma, float *out,
                                const float *state_in, float *state_out,
                                int B, int H, int N, int d, int dtype, int mask, void *stream);

/*
 * Rank different from the value width.  The operator is defined for B, C in R^(N x r) and
 * V in R^(N x d) (Section 2.2); the entry points above take r = d.  These take them apart:
 *   q, k   [B][H][N][r]      v, out   [B][H][N][dv]      states   [B][H][r][dv] float
 * Supported: r = dv in {64, 128} for every input type, and r = 128, dv = 256 (the shape of the
 * paper's usage example, Section 4) for LEET_BF16 and LEET_F16 inputs; anything else returns
 * LEET_ERR_UNSUPPORTED.  All other arguments as in leet_attn_forward_v2,
 * leet_attn_forward_recurrent, leet_attn_decode_step_v2 and leet_attn_workspace_bytes.
 */
int leet_attn_forward_rd(const void *q, const void *k, const void *v, const float *gamma, void *out,
                         const float *state_in, float *state_out,
                         void *workspace, size_t workspace_bytes, int segments,
                         int B, int H, int N, int r, int dv, int in_dtype, int out_dtype, int mask, void *stream);
int leet_attn_forward_recurrent_rd(const void *q, const void *k, const void *v, const float *gamma, float *out,
                                   const float *state_in, float *state_out,
                                   int B, int H, int N, int r, int dv, int dtype, int mask, void *stream);
int leet_attn_decode_step_rd(const void *q, const void *k, const void *v, const float *gamma,
                             float *state_inout, float *out, int B, int H, int r, int dv, int dtype, int mask,
                             void *stream);
size_t leet_attn_workspace_bytes_rd(int B, int H, int N, int r, int dv, int dtype, int segments);

/*
 * FleetAttention prefill: the operator as the sum over the rank of discounted cumulative sums,
 * O = sum_j diag(b_j) lambda-cumsum(diag(c_j) V) (Section 3, Eq. "p"; Appendix C.1 for the decay),
 * evaluated in column blocks (parallel) and row blocks (in order) with one carried vector per
 * rank index, as Alg. 5 (Appendix B.4) lays it out.  Element-wise work on the vector ALUs only,
 * no MFMA: like the row-based kernel it is an in-library comparison point (the paper's own
 * measurements, Section 5.1 and Appendix E, have it slowest), not the fast path.
 *   q, k   [B][H][N][r] of `dtype` (the paper's B and C)      v   [B][H][N][dv] of `dtype`
 *   out    [B][H][N][dv] float
 *   state_in, state_out   [B][H][r][dv] float or NULL: the carried vectors l^j entering the first
 *          row block and leaving the last; they are the rows of the state the other kernels use
 *   mask   a leet_mask (gamma may be NULL for LEET_MASK_CAUSAL: plain cumsum)
 * Shapes as for leet_attn_forward_recurrent_rd.  Needs no workspace and no atomics.
 */
int leet_attn_forward_fleet(const void *q, const void *k, const void *v, const float *gamma, float *out,
                            const float *state_in, float *state_out,
                            int B, int H, int N, int r, int dv, int dtype, int mask, void *stream);

/* As leet_attn_decode_step_ex, with `dtype` also LEET_F16 and with a leet_mask. */
int leet_attn_decode_step_v2(const void *q, const void *k, const void *v, const float *gamma,
                             float *state_inout, float *out, int B, int H, int d, int dtype, int mask,
                             void *stream);

/*
 * Bytes of workspace leet_attn_forward_ex needs for this shape with `segments`
 * as above (0 = library's choice) under the process-wide kernel choice: one d x d
 * fp32 state per segment boundary the library computes, plus one per sequence for
 * the copy of the entering state.  Returns 0 when no workspace is needed (one
 * segment) or the arguments are invalid.
 */
size_t leet_attn_workspace_bytes(int B, int H, int N, int d, int dtype, int segments);

/*
 * Frees the library-owned workspace of the current device, including blocks retired
 * when it grew (synchronises the device first).  Optional; the workspace is
 * otherwise kept until process exit.  A graph captured from a call that used the
 * library-owned workspace must not be replayed after this.
 */
int leet_attn_release_workspace(void);

/*
 * Tuning knob: which kernel a bf16 or fp16 prefill uses.  Both compute the same chunked form (Alg. 2
 * with the decaying mask) and pass the same parity tests; they differ in how the work is split.
 *   LEET_KERNEL_WIDE          one workgroup per (sequence, segment), all d value columns
 *   LEET_KERNEL_COLUMN_SPLIT  dv/32 workgroups per (sequence, segment), 32 value columns each,
 *                             placed on one XCD; fewer segments needed to fill the device
 *                             (16-bit inputs, every supported shape; fp32 runs wide)
 *   LEET_KERNEL_AUTO          (default) the library prices both kernels at each candidate segment
 *                             count with a cost model fitted to measurements and takes the
 *                             cheapest pair; leet_attn_query_plan reports the outcome
 * With WIDE or COLUMN_SPLIT set, only the segment count is chosen that way.
 * The setter changes the process-wide default, which every entry point without a `kernel`
 * argument uses; a thread that must not depend on what other threads set between its workspace
 * query and its call passes the choice per call (the _v3 entry points below).  Returns
 * LEET_ERR_INVALID_ARG for any other value.
 */
typedef enum { LEET_KERNEL_WIDE = 0, LEET_KERNEL_COLUMN_SPLIT = 1, LEET_KERNEL_AUTO = 2 } leet_bf16_kernel;
int leet_attn_set_bf16_kernel(int which);
int leet_attn_get_bf16_kernel(void);

/*
 * Tuning knob: how a decode step stores the updated state.
 *   LEET_DECODE_STORE_AUTO    (default) a state under a quarter of the 256 MB last-level cache is
 *                             cached.  A larger one is cached only when it is being stepped alone --
 *                             the previous decode call on this device updated this very buffer, and
 *                             it fits half of the cache -- and streamed otherwise (another state came
 *                             in between, or this is its first step).  Streaming a state that would
 *                             have stayed cached costs about 5 %, caching one that is displaced
 *                             before its next step about 20 %
 *   LEET_DECODE_STORE_CACHED  ordinary stores: best when the next step on the same state finds it
 *                             in the cache (one small model stepping alone)
 *   LEET_DECODE_STORE_STREAM  nontemporal stores: best when other states are touched before this one
 *                             is used again (many layers taking turns), whatever its size
 * The results are identical; only the memory traffic differs.  The setter changes the
 * process-wide default; leet_attn_decode_step_v3 takes the policy per call.
 */
typedef enum { LEET_DECODE_STORE_AUTO = 0, LEET_DECODE_STORE_CACHED = 1, LEET_DECODE_STORE_STREAM = 2 } leet_decode_store;
int leet_attn_set_decode_store(int mode);
int leet_attn_get_decode_store(void);

/*
 * Every choice per call.  `kernel` is a leet_bf16_kernel value and `store` a leet_decode_store
 * value, or LEET_CHOICE_DEFAULT for the process-wide setting; everything else as in
 * leet_attn_forward_rd, leet_attn_workspace_bytes_rd, leet_attn_query_plan_rd and
 * leet_attn_decode_step_rd.  A caller that passes the same `kernel` and `segments` to
 * leet_attn_workspace_bytes_v3 and to leet_attn_forward_v3 gets a workspace size that matches
 * the call whatever other threads do with the setters.
 */
#define LEET_CHOICE_DEFAULT (-1)
int leet_attn_forward_v3(const void *q, const void *k, const void *v, const float *gamma, void *out,
                         const float *state_in, float *state_out,
                         void *workspace, size_t workspace_bytes, int segments, int kernel,
                         int B, int H, int N, int r, int dv, int in_dtype, int out_dtype, int mask, void *stream);
size_t leet_attn_workspace_bytes_v3(int B, int H, int N, int r, int dv, int dtype, int segments, int kernel);
int leet_attn_query_plan_v3(int B, int H, int N, int r, int dv, int dtype, int segments, int kernel_choice,
                            int *nseg, int *kernel);
int leet_attn_decode_step_v3(const void *q, const void *k, const void *v, const float *gamma,
                             float *state_inout, float *out, int B, int H, int r, int dv, int dtype, int mask,
                             int store, void *stream);

/*
 * What leet_attn_forward_ex would do for this shape under the current kernel choice (fp32
 * output, decaying mask; the plan depends on neither): *nseg receives the number of segments per
 * sequence, *kernel LEET_KERNEL_WIDE or LEET_KERNEL_COLUMN_SPLIT (fp32 inputs always run WIDE;
 * both 16-bit types have both kernels).  Either pointer may be NULL.  Host-only; touches no device.
 */
int leet_attn_query_plan(int B, int H, int N, int d, int dtype, int segments, int *nseg, int *kernel);
/* The same for rank r and value width dv given separately (shapes as for leet_attn_forward_rd). */
int leet_attn_query_plan_rd(int B, int H, int N, int r, int dv, int dtype, int segments, int *nseg, int *kernel);

/*
 * Backward pass of the prefill: gradients of q, k, v and of the entering state from that of the output,
 *     dq_i = sum over j <= i of gamma^(i-j) (dout_i . v_j) k_j  +  gamma^(i+1) state_in dout_i,
 *     dk_j = sum over i >= j of gamma^(i-j) (v_j . dout_i) q_i  +  gamma^(N-1-j) dstate_out v_j,
 *     dv_j = sum over i >= j of gamma^(i-j) (k_j . q_i) dout_i  +  gamma^(N-1-j) k_j dstate_out,
 *     dstate_in = sum over i of gamma^(i+1) q_i^T dout_i  +  gamma^N dstate_out.
 * The scores are formed again, nothing of the forward call has to be kept but its inputs.  gamma is a fixed number a head
 * (as in the paper) and has no gradient.
 *   dout         [B][H][N][dv] of `dtype`: the gradient of `out`.  A 16-bit call's gradient is taken in 16 bits whatever the
 *                forward call's out_dtype was
 *   q, k, v      what the forward call was given
 *   dq, dk, dv_out  [B][H][N][r], [B][H][N][r], [B][H][N][dv] of `dtype`, rounded once, at the store
 *   state_in     what the forward call was given ([B][H][r][dv] float or NULL)
 *   dstate_out   the gradient of its state_out, or NULL: zero
 *   dstate_in    [B][H][r][dv] float or NULL: not wanted
 *   workspace    leet_attn_backward_workspace_bytes bytes for the same `segments`, 256-byte aligned (NULL when that is 0);
 *                always the caller's, so calls on several streams and captured graphs share nothing.  Scratch
 *   segments     as for leet_attn_forward_ex
 * Shapes as for leet_attn_forward_rd, `dtype` any leet_dtype, `mask` a leet_mask (gamma may be NULL for LEET_MASK_CAUSAL).
 * Inside, scores and, as operands of products, states are rounded to the input type, as in the forward pass (of at most 128
 * tokens to twice its bits), in fp16 times powers of two that keep them within its range, whatever the inputs' size: gradients
 * are infinite only where they themselves leave their type.  States are carried in fp32, and dstate_in is exact to fp32's
 * products (in fp16 to those of a q whose numbers below 2^-14 count as 2^-14).  A value that is not finite may make all
 * gradients of its sequence so.
 * Outputs and workspace that share memory with one another or with an input are LEET_ERR_INVALID_ARG.  N = 0 is legal and
 * hands the state's gradient on.
 */
int leet_attn_backward(const void *dout, const void *q, const void *k, const void *v, const float *gamma,
                       void *dq, void *dk, void *dv_out, const float *state_in, const float *dstate_out, float *dstate_in,
                       void *workspace, size_t workspace_bytes, int segments,
                       int B, int H, int N, int r, int dv, int dtype, int mask, void *stream);
size_t leet_attn_backward_workspace_bytes(int B, int H, int N, int r, int dv, int dtype, int segments);

/* ------------------------------------------------------------------------------------------------
 * Operators beside the attention: what makes its queries and keys (position rotation, norms of each
 * head), the element-wise recurrence with a decay of its own for every token and channel, norms of a
 * residual stream, and the clipping of a model's gradients.
 * Of the conventions above these differ: tensors may have strides (in ELEMENTS; the elements of a
 * head row, or the channels of a token row, are adjacent), pointers need only their element's
 * alignment, and a workspace, where one is needed, is always the caller's, so that calls on several
 * streams and captured graphs share nothing.  Calls that may overlap in time need one each (the
 * recurrence's workgroups find one another through it).  Outputs and workspaces that share memory with
 * one another or with an input, other than in place where a call says so, are LEET_ERR_INVALID_ARG.
 * (Rows of one buffer may lie between one another.  Where the strides leave more possibilities than the
 * check looks at, which parts of one buffer at the same strides never do, the call is not refused.)
 * N = 0 is legal everywhere here and writes no rows.
 * ---------------------------------------------------------------------------------------------- */

/* Element (b, h, n, j) of a [B][H][N][d] tensor is at data + b*batch + h*head + n*token + j.  A
 * [B][N][H][d] projection is such a view, and so is a part of a wider one.  Rows that are written
 * must not overlap one another (LEET_ERR_INVALID_ARG for strides that do not keep them apart). */
typedef struct {
    void *data;
    long long batch, head, token;
} leet_attn_heads;

typedef enum {
    LEET_ROPE_HALF = 0,       /* element i of the rotated part is paired with i + rot/2 */
    LEET_ROPE_INTERLEAVED = 1 /* elements 2i and 2i + 1 are paired                      */
} leet_rope_layout;

/*
 * Position rotation: pair i of the first `rot` elements of a head row at position p is turned by
 * theta = p freq[i] and multiplied by `scale`,
 *     y1 = scale (x1 cos theta - x2 sin theta),   y2 = scale (x2 cos theta + x1 sin theta);
 * the elements from `rot` on are passed on.  Angles, cosines and sines are formed in fp64, these times
 * the scale rounded to fp32 once.  An angle is off by some 2^-52 of itself, half a step of fp32 at 2^27
 * radians; positions farther out are turned by less and less certain angles.
 *   freq       [rot/2] double, DEVICE memory: radians a position
 *   rot        even, 2 <= rot <= d
 *   positions  NULL: token n is at pos0 + n; else 64-bit integers, token n of sequence b at
 *              positions[b*positions_batch + n] (positions_batch 0: the same for every sequence);
 *              pos0 is added
 *   scale      finite; 1 but for contexts stretched by bands
 */
typedef struct {
    const double *freq;
    int rot;
    int layout; /* a leet_rope_layout */
    const long long *positions;
    long long positions_batch, pos0;
    float scale;
} leet_attn_rotation;

/* How a table of frequencies is made for contexts longer than the trained one. */
typedef enum {
    LEET_ROPE_SCALING_NONE = 0,   /* f_i = base^(-2i/rot)                                          */
    LEET_ROPE_SCALING_LINEAR = 1, /* f_i / factor: positions squeezed into the trained range       */
    LEET_ROPE_SCALING_BASE = 2,   /* base factor^(rot/(rot-2)): the slowest pair is stretched by
                                     factor, the fastest not at all (rot = 2: no scaling)          */
    LEET_ROPE_SCALING_BANDS = 3,  /* pairs that turn over `fast` times within the trained length
                                     keep f_i, those under `slow` times get f_i / factor, with a
                                     ramp over the pair's index between the two (its ends rounded
                                     outward to whole indices); *scale = 0.1 ln(factor) + 1        */
    LEET_ROPE_SCALING_TURNS = 4   /* the same two ends with the ramp over the number of turns
                                     within the trained length; *scale = 1                         */
} leet_rope_scaling;

/* Fills freq[rot/2] and *scale (HOST memory, in fp64).  base > 1, factor >= 1; `trained` (tokens) > 0
 * and 0 < slow < fast for BANDS and TURNS, ignored otherwise.  Touches no device. */
int leet_attn_rope_frequencies(int rot, double base, int scaling, double factor, int trained, double slow,
                               double fast, double *freq, float *scale);

/*
 * Position rotation of queries and, in the same launch, of keys.
 *   q, k          [B][Hq][N][d], [B][Hk][N][d] of `dtype`; k and out_k may be NULL (Hk is then ignored)
 *   out_q, out_k  of the same shapes and type; each may be its input itself (same data and strides)
 *   transposed    non-zero: the transposed map (angles negated, same scale), which takes gradients of
 *                 the outputs to gradients of the inputs
 * d even, 2 <= d <= 256.  Rounded once, at the store.
 */
int leet_attn_rope(const leet_attn_heads *q, const leet_attn_heads *out_q, int Hq,
                   const leet_attn_heads *k, const leet_attn_heads *out_k, int Hk,
                   const leet_attn_rotation *rotation, int B, int N, int d, int dtype, int transposed,
                   void *stream);

/*
 * Norm of every query and key head, then the rotation, in one pass:
 *     y = R (w .* x / sqrt(mean(x^2) + eps)).
 *   q_weight, k_weight  [d] of weight_dtype (`dtype` or LEET_F32), or NULL: ones
 *   eps                 >= 0, finite.  A row of zeros with eps = 0 gives NaN, as the formula does
 * The rest as for leet_attn_rope; fp32 inside, rounded once, at the store.  A row whose squares would leave
 * fp32's range is multiplied by a power of two for its norm, so any finite row has one.
 */
int leet_attn_qk_norm_rope(const leet_attn_heads *q, const leet_attn_heads *out_q, int Hq,
                           const leet_attn_heads *k, const leet_attn_heads *out_k, int Hk,
                           const void *q_weight, const void *k_weight, int weight_dtype, float eps,
                           const leet_attn_rotation *rotation, int B, int N, int d, int dtype, void *stream);

/*
 * Its backward pass, from the same inputs and the gradients of the outputs.  With u = R^T dy,
 * r = 1/sqrt(mean(x^2) + eps) and n = x r:
 *     dx = r (w .* u - n mean(w .* u .* n)),      dw = sum of u .* n over tokens and heads.
 *   dout_q, dout_k        gradients of the outputs
 *   dq, dk                gradients of the inputs; each may be the gradient it comes from, or the input
 *                         (same data and strides)
 *   dq_weight, dk_weight  [d] of weight_dtype, two of them, or NULL: not wanted.  Written when all inputs
 *                         have been read, so each may be its weight
 *   workspace             leet_attn_qk_norm_rope_workspace_bytes bytes, 256-byte aligned; may be NULL
 *                         when neither weight's gradient is wanted.  Its contents are scratch
 * The sums over tokens and heads are taken in fp32 in a fixed order: no atomics, equal from call to call.
 */
int leet_attn_qk_norm_rope_backward(const leet_attn_heads *dout_q, const leet_attn_heads *q,
                                    const leet_attn_heads *dq, int Hq,
                                    const leet_attn_heads *dout_k, const leet_attn_heads *k,
                                    const leet_attn_heads *dk, int Hk,
                                    const void *q_weight, const void *k_weight, void *dq_weight, void *dk_weight,
                                    int weight_dtype, float eps, const leet_attn_rotation *rotation,
                                    void *workspace, size_t workspace_bytes,
                                    int B, int N, int d, int dtype, void *stream);
size_t leet_attn_qk_norm_rope_workspace_bytes(int B, int Hq, int Hk, int N, int d);

/*
 * Gated linear recurrence, element-wise in every channel:
 *     h_t = a_t h_{t-1} + b_t,
 * with a_t, b_t from the gate z_t and the input x_t by `mode`.  (A decay that is one constant a head
 * makes it the discounted cumulative sum that leet_attn_forward_fleet takes per rank.)
 */
typedef enum {
    LEET_GATE_DECAY = 0,  /* a = z,           b = x                                         */
    LEET_GATE_LOG = 1,    /* a = exp(z),      b = x                                         */
    LEET_GATE_SIGMOID = 2 /* a = sigmoid(z),  b = (1 - a) x: h is a moving average of x     */
} leet_gate_mode;

/* Element (b, n, c) of a [B][N][C] tensor is at data + b*batch + n*token + c. */
typedef struct {
    void *data;
    long long batch, token;
} leet_attn_rows;

/*
 * Over whole sequences.
 *   x, out     [B][N][C] of `dtype`;  gate  [B][N][C] of gate_dtype (`dtype` or LEET_F32)
 *   out        h of every token, rounded once, at the store (the recurrence itself runs in fp32)
 *   state_in   [S][C] float or NULL (zeros): h before each sequence's first token
 *   state_out  [S][C] float or NULL; receives h after each sequence's last token; may be state_in
 *   offsets    NULL: every batch entry is one sequence of N tokens, S = B (`sequences` is ignored).
 *              Else DEVICE memory, sequences + 1 ints, not falling, offsets[0] = 0 and
 *              offsets[S] <= N: the sequences lie behind one another in the N rows, sequence s in rows
 *              offsets[s] .. offsets[s+1]-1, with B = 1.  Empty sequences hand their state on.  Rows
 *              from offsets[S] on are not read for a result and their outputs are left as they were.
 *              (The values are not diagnosed; other ones give wrong rows but no access out of range.)
 *   workspace  leet_attn_gated_scan_workspace_bytes bytes, 256-byte aligned (NULL when that is 0); scratch
 * Decays may have any values.  Tokens are combined in tiles of up to 240 tokens and 128 channels by the
 * products of their decays, formed in fp32: of the state that enters a tile nothing is left where that
 * product is under 2^-149.  A tile in which decays above 1 in magnitude multiply to more than 16 within some
 * sixteen tokens is taken token by token from the state before it instead, and the tiles behind it wait: the
 * recurrence as it stands, at 5 to 30 times the time where every tile does (the longer the sequences and the
 * fewer the channels, the slower).  A non-finite value makes the later values of its
 * channel and sequence non-finite and no others (once such a state has decayed to nothing it is NaN).
 */
int leet_attn_gated_scan(const leet_attn_rows *x, const leet_attn_rows *gate, const leet_attn_rows *out,
                         const float *state_in, float *state_out, const int *offsets, int sequences,
                         void *workspace, size_t workspace_bytes,
                         int B, int N, int C, int dtype, int gate_dtype, int mode, void *stream);

/*
 * Its backward pass.  h is the forward call's output; with dh the gradient of h,
 *     D_t = dh_t + g_{t+1},   g_t = a_t D_t,   g behind the last token = dstate_out (zero if NULL),
 *     dx = D (times 1 - a for LEET_GATE_SIGMOID),
 *     dgate = D h_{t-1} | g h_{t-1} | D (h_{t-1} - x) a (1 - a)      by mode,
 *     dstate_in = g of the first token.
 *   x            read by LEET_GATE_SIGMOID only; may be NULL otherwise
 *   h, dh, dx    [B][N][C] of `dtype`;  dgate  of gate_dtype
 *   state_in     what the forward call was given (NULL: zeros)
 *   dstate_out   [S][C] float or NULL;  dstate_in  [S][C] float or NULL; may be dstate_out
 * The rest as for leet_attn_gated_scan.
 */
int leet_attn_gated_scan_backward(const leet_attn_rows *dh, const leet_attn_rows *x, const leet_attn_rows *gate,
                                  const leet_attn_rows *h, const leet_attn_rows *dx, const leet_attn_rows *dgate,
                                  const float *state_in, const float *dstate_out, float *dstate_in,
                                  const int *offsets, int sequences, void *workspace, size_t workspace_bytes,
                                  int B, int N, int C, int dtype, int gate_dtype, int mode, void *stream);
size_t leet_attn_gated_scan_workspace_bytes(int B, int N, int C, int backward);

/*
 * One token of every sequence: state <- a state + b, out = state (rounded).
 *   x, gate, out  [B][C], row b at data + b*batch (`token` is ignored);  state  [B][C] float, in place
 *   out may be x, or a gate of its type (same data and stride)
 */
int leet_attn_gated_scan_step(const leet_attn_rows *x, const leet_attn_rows *gate, const leet_attn_rows *out,
                              float *state, int B, int C, int dtype, int gate_dtype, int mode, void *stream);

/*
 * Root-mean-square norm of rows, the residual stream's addition in the same pass:
 *     s = x + residual,     out = w .* s / sqrt(mean(s^2) + eps),     residual_out = s.
 *   x, out        [B][N][C] of `dtype`
 *   residual, residual_out  [B][N][C] of residual_dtype (`dtype` or LEET_F32); residual NULL: s = x, and residual_out must be
 *                 NULL; residual_out NULL: not wanted
 *   weight        [C] of weight_dtype (`dtype` or LEET_F32), or NULL: ones
 *   eps           >= 0, finite.  A row of zeros with eps = 0 gives NaN, as the formula does
 * The norm is that of the sum before it is rounded to residual_dtype.  fp32 inside, rounded once, at the store; a row whose
 * squares would leave fp32's range is multiplied by a power of two for its norm.  out may be x or residual, residual_out
 * residual or x (same data, strides and type).  C <= 16384 (LEET_ERR_TOO_LARGE).
 */
int leet_attn_add_rms_norm(const leet_attn_rows *x, const leet_attn_rows *residual, const leet_attn_rows *out,
                           const leet_attn_rows *residual_out, const void *weight, int weight_dtype, float eps,
                           int B, int N, int C, int dtype, int residual_dtype, void *stream);

/*
 * The same with an output in 8 bits (e4m3: four bits of exponent, three of mantissa, largest value 448) and scales:
 *     scale = max(largest |y|, 2^-100) / 448,     out = e4m3(y / scale),     y = out scale.
 *   out      [B][N][C] bytes (strides in bytes)
 *   scales   [B][N][C / group] float, dense; one for `group` neighbouring channels: 32, 64 or 128, which must divide C, or 0:
 *            one a row, scales [B][N]
 * Where y is not a finite number the row's or group's scale or values are not either.
 */
int leet_attn_add_rms_norm_q8(const leet_attn_rows *x, const leet_attn_rows *residual, const leet_attn_rows *out,
                              float *scales, int group, const leet_attn_rows *residual_out, const void *weight,
                              int weight_dtype, float eps, int B, int N, int C, int dtype, int residual_dtype, void *stream);

/*
 * Backward pass of leet_attn_add_rms_norm.  With r = 1/sqrt(mean(h^2) + eps) and n = h r:
 *     g = r (w .* dout - n mean(w .* dout .* n)) + dresidual,     dweight = sum of dout .* n over the rows;
 * g is the gradient of the sum, so of x and of the residual both.
 *   dout       [B][N][C] of `dtype`: the gradient of out
 *   h          [B][N][C] of residual_dtype: the forward call's residual_out (x where there was no residual)
 *   dresidual  [B][N][C] of residual_dtype: the gradient of residual_out, or NULL: zero
 *   dx, dh     g in `dtype`, g in residual_dtype; either may be NULL.  Each may be dout, h or dresidual (same data, strides and type)
 *   dweight    [C] of weight_dtype, or NULL: not wanted.  Written when all inputs have been read, so it may be the weight
 *   workspace  leet_attn_add_rms_norm_workspace_bytes bytes, 256-byte aligned; may be NULL without dweight.  Scratch
 * The sums over rows are taken in fp32 in a fixed order: no atomics, equal from call to call.  Products of w, dout and h have to
 * stay within fp32's range.
 */
int leet_attn_add_rms_norm_backward(const leet_attn_rows *dout, const leet_attn_rows *h, const leet_attn_rows *dresidual,
                                    const leet_attn_rows *dx, const leet_attn_rows *dh, const void *weight, void *dweight,
                                    int weight_dtype, float eps, void *workspace, size_t workspace_bytes,
                                    int B, int N, int C, int dtype, int residual_dtype, void *stream);
size_t leet_attn_add_rms_norm_workspace_bytes(int B, int N, int C);

/* One of a model's gradients: `count` adjacent values of `dtype`, DEVICE memory, and where the clipped ones go (may be data). */
typedef struct {
    const void *data;
    void *out;
    long long count;
    int dtype;
} leet_attn_gradient;

/*
 * The norm over all gradients of a model, and the gradients clipped to it:
 *     norm = sqrt(sum of all squares),     out = data min(1, limit / norm).
 *   grads      HOST memory, read before the call returns; `count` of them, of any types and sizes (0 values are legal)
 *   limit      >= 0; INFINITY: the norm alone, `out` is ignored
 *   norm       one float, DEVICE memory, or NULL: not wanted
 *   workspace  leet_attn_clip_gradients_workspace_bytes bytes, 256-byte aligned; scratch
 * Squares are added in fp64 in a fixed order, so the norm neither overflows (but as a float) nor changes from call to call.  A
 * norm that is not finite clips nothing: `out` then holds the gradients as they are.  Where nothing is clipped gradients in
 * place are not written.
 */
int leet_attn_clip_gradients(const leet_attn_gradient *grads, int count, float limit, float *norm, void *workspace,
                             size_t workspace_bytes, void *stream);
size_t leet_attn_clip_gradients_workspace_bytes(void);

/* Static, never-NULL description of a leet_status value. */
const char *leet_attn_strerror(int status);

/* Library version as "major.minor.patch". */
const char *leet_attn_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LEET_ATTN_H */
