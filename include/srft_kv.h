/*
 * srft_kv.h -- C ABI of the fused SRFT int4 KV-cache quantizer for AMD MI355X (gfx950).
 *
 * Write path (paper Sec. 3.2 steps 1-4, Sec. 5.1 item 1, Sec. 7.1), per head-dim vector x in fp16:
 *     u = s * x                      s in {-1,+1}^d, fixed per plan                       (Eq. 1)
 *     z = pack(F u)                  F the unitary DFT, real packing of Eq. 2             (Eq. 1-2)
 *     w = lambda * z                 per-channel rescale                                  (Sec. 5.1)
 *     scale_j = max_{k in group j} |w_k| / 7,  groups = runs of g packed indices          (Sec. 7.1)
 *     q_k = rint(w_k / scale_j) in [-7, 7]   (round half to even)                         (Sec. 3.2 step 4)
 *     byte_i = (q_{2i+1} << 4) | (q_{2i} & 0xF)                                           (Sec. 3.2 (ii))
 * Read path (the inverse kernel of Sec. 7.1): unpack nibbles (4-bit two's complement), times
 * scale_j, divide by max(lambda_k, 1e-6), unpack Eq. 2, unitary inverse DFT, times s, round to fp16.
 *
 * Stored record per vector: d/2 code bytes and d/g fp32 scales, in two separate arrays.
 *
 * Conventions
 *   - "dev" pointers are device (HBM) addresses on the GPU that was current when the plan was
 *     created; "host" pointers are ordinary host memory.  The caller owns every buffer it passes;
 *     the library allocates only the plan's own constant tables, which srft_plan_destroy frees, and a
 *     256 KB table of all plans of a device, which goes with the last of them.
 *   - Calls that take a stream enqueue on it and return without synchronising.  hip_stream is a
 *     hipStream_t passed as void* (NULL = the default stream).
 *   - Every function returns SRFT_OK (0) or a negative srft_status; nothing aborts or throws.
 *     All argument checks happen before the first HIP call.
 *   - Supported shapes: d a multiple of 32 with 32 <= d <= 256 (so 96 = 2^5 * 3 is covered; the
 *     transform is applied as a dense d x d contraction, which needs no power-of-two length);
 *     group_size g = 32 (the deployed format, the fast path), 16, or any multiple of 32 that divides d
 *     (g = d is the per-token quantizer of Sec. 3.2 step 3).
 */
#ifndef SRFT_KV_H
#define SRFT_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct srft_plan srft_plan_t;   /* opaque; owned by the library */

typedef enum srft_status {
    SRFT_OK             =  0,
    SRFT_ERR_NULL       = -1,   /* a required pointer is NULL */
    SRFT_ERR_BAD_D      = -2,   /* d not a multiple of 32 in [32, 256] */
    SRFT_ERR_BAD_GROUP  = -3,   /* group_size not 16 and not a multiple of 32 dividing d */
    SRFT_ERR_BAD_LAMBDA = -4,   /* a lambda is not finite, not > 0, or max/min exceeds 2^16 */
    SRFT_ERR_ALIGN      = -5,   /* a device pointer is not aligned as documented */
    SRFT_ERR_HIP        = -6,   /* a HIP call failed; see srft_last_hip_error() */
    SRFT_ERR_BAD_N      = -7,   /* n_vec < 0, count < 0 or byte count negative */
    SRFT_ERR_MISMATCH   = -8,   /* plans of one call differ in d, group_size, code width or device */
    SRFT_ERR_BAD_BITS   = -9,   /* code width not 4 or 8 */
    SRFT_ERR_BAD_TRANSFORM = -10 /* transform not one of srft_transform */
} srft_status;

/*
 * Build a plan: the constants of one (layer, K|V) pair.                 (Eq. 1; Sec. 5.1; Sec. 7.1-7.2)
 *   out          receives the plan (host pointer to a host pointer).
 *   d            head dimension.
 *   group_size   g, the number of consecutive packed indices sharing one scale.
 *   sign_seed    the sign diagonal is the splitmix64 stream started at this seed: s_n = -1 iff the
 *                top bit of the n-th output is set (the signs are fixed when the plan is made, Sec. 3.1).
 *   lambda_host  d floats > 0 on the host, or NULL for all ones.  Copied; not kept.
 * Allocates device tables on the current GPU (12*d*d to 16*d*d bytes) and copies them once.
 */
int srft_plan_create(srft_plan_t** out, int d, int group_size, uint64_t sign_seed,
                     const float* lambda_host);

/*
 * The same with a chosen code width.                                   (Sec. 3.2 steps 3-4: b in {4, 8})
 *   bits = 4   the format above (srft_plan_create is this case).
 *   bits = 8   scale_j = max |w_k| / 127, q_k = rint(w_k / scale_j) in [-127, 127], one two's-complement byte per
 *              value: codes are [n_vec, d] bytes, byte k = q_k; the record is d + 4 d/g bytes.  Every entry point
 *              that takes codes then takes this layout (srft_plan_code_bytes tells the row size).
 */
int srft_plan_create_bits(srft_plan_t** out, int d, int group_size, int bits, uint64_t sign_seed,
                          const float* lambda_host);

/*
 * The same with a chosen mixing matrix: the comparator of Sec. 1 / Sec. 3.1.
 *   SRFT_TRANSFORM_DFT       the real-packed unitary DFT of Eq. 1-2 (every other create call is this case).
 *   SRFT_TRANSFORM_HADAMARD  the orthonormal Walsh-Hadamard matrix in natural order, H[k][n] = (-1)^popcount(k & n)
 *                            / sqrt(d): sign diagonal, lambda, quantizer and record are unchanged, which makes the
 *                            pipeline the SRHT the paper compares against.  d must be a power of two (else
 *                            SRFT_ERR_BAD_D).  Runs on the plain kernels (the folded forms use DFT symmetries).
 */
typedef enum srft_transform { SRFT_TRANSFORM_DFT = 0, SRFT_TRANSFORM_HADAMARD = 1 } srft_transform;
int srft_plan_create_ex(srft_plan_t** out, int d, int group_size, int bits, int transform, uint64_t sign_seed,
                        const float* lambda_host);

/* Free the plan and its device tables.  NULL is accepted.  Work already enqueued must have finished. */
int srft_plan_destroy(srft_plan_t* plan);

/*
 * Write path over n_vec vectors.                                        (Sec. 3.2 steps 1-4, Sec. 7.1)
 *   x_f16_dev   [n_vec, d] row-major IEEE fp16, 16-byte aligned.        read only
 *   codes_dev   [n_vec, d/2] bytes ([n_vec, d] for an 8-bit plan), 16-byte aligned.   written
 *   scales_dev  [n_vec, d/g] fp32, 4-byte aligned.                      written
 * n_vec == 0 is a successful no-op; n_vec > 2^33 is SRFT_ERR_BAD_N (tile indices are 32-bit).  Inputs must be finite.  A group whose abs-max / 7 is below
 * 2^-100 is stored as scale 0 with all-zero codes.
 */
int srft_kv_quantize(const srft_plan_t* plan, const void* x_f16_dev, int64_t n_vec,
                     uint8_t* codes_dev, float* scales_dev, void* hip_stream);

/*
 * Read path over n_vec vectors: the inverse of srft_kv_quantize.        (Sec. 7.1; sentence after Eq. 2)
 *   codes_dev   [n_vec, d/2] bytes ([n_vec, d] for an 8-bit plan), 16-byte aligned.   read only
 *   scales_dev  [n_vec, d/g] fp32, 4-byte aligned.                      read only
 *   out_f16_dev [n_vec, d] fp16 (round to nearest even), 16-byte aligned.  written
 * Nibble 0x8 decodes as -8 (byte 0x80 as -128 at 8 bits).
 */
int srft_kv_dequantize(const srft_plan_t* plan, const uint8_t* codes_dev, const float* scales_dev,
                       int64_t n_vec, void* out_f16_dev, void* hip_stream);

/*
 * Write path / read path over several plans in one launch.     (Sec. 7.2: one stored transform per layer and
 * K|V; a decode step appends a few vectors to every one of them, so a launch per plan is all latency.)
 *   plans, *_dev arrays, n_vec   HOST arrays of `count` entries; entry i describes one call of
 *                                srft_kv_quantize / srft_kv_dequantize (same shapes, alignment and ownership;
 *                                the *_dev entries are device addresses).  The arrays are read before the call
 *                                returns and not kept.
 *   count                        number of entries; 0 is a successful no-op.  Entries with n_vec[i] == 0 are
 *                                skipped (their pointers are not looked at).
 * All plans must share d, group_size, code width, transform and device (else SRFT_ERR_MISMATCH); signs and lambda
 * may differ.
 * Every entry is validated before anything is enqueued.  Up to 64 entries go into one kernel launch; longer
 * lists take several launches on the same stream.  Results are bit-identical to the per-plan calls.
 * Buffers of different entries must not overlap.
 */
int srft_kv_quantize_batched(const srft_plan_t* const* plans, const void* const* x_f16_dev,
                             const int64_t* n_vec, uint8_t* const* codes_dev, float* const* scales_dev,
                             int count, void* hip_stream);
int srft_kv_dequantize_batched(const srft_plan_t* const* plans, const uint8_t* const* codes_dev,
                               const float* const* scales_dev, const int64_t* n_vec,
                               void* const* out_f16_dev, int count, void* hip_stream);

/*
 * The write path with the transform done as FFT butterflies on the vector ALU, in fp32: a complex FFT of half the
 * length and a Hermitian unpack (Sec. 3.2; the form of the kernel of Sec. 7.1) in place of the matrix-core contraction
 * that srft_kv_quantize uses.  Same arguments and the same record, except that scales_dev must be 16-byte aligned; for
 * plans with d = 128 or 256, g = 32, 4-bit codes and the DFT (else SRFT_ERR_BAD_D / _BAD_GROUP / _BAD_BITS /
 * _BAD_TRANSFORM).  At d = 128 a lane holds a whole vector; at d = 256 two lanes share one and exchange
 * registers.
 * It exists so that the two forms can be timed side by side (bench.py --butterfly); it is the slower one on this
 * machine, and codes may differ from srft_kv_quantize's where a value sits at a rounding boundary.
 */
int srft_kv_quantize_butterfly(const srft_plan_t* plan, const void* x_f16_dev, int64_t n_vec,
                               uint8_t* codes_dev, float* scales_dev, void* hip_stream);

/*
 * The transform alone, quantization disabled: w = lambda * pack(F (s * x)) in fp32.  (Eq. 1-2, Sec. 5.1)
 *   x_f16_dev [n_vec, d] fp16, 16-byte aligned; w_f32_dev [n_vec, d] fp32, 16-byte aligned, written.
 * Same kernel as the write path up to the abs-max; exists so that the transform can be checked
 * on its own (orthonormality, closed forms).
 */
int srft_kv_forward_f32(const srft_plan_t* plan, const void* x_f16_dev, int64_t n_vec,
                        float* w_f32_dev, void* hip_stream);

/*
 * Scores of queries against stored keys, without reconstructing the keys.    (Sec. 1: the decode step streams the
 * stored prefix before attention reads it; Eq. 1 and the sentence after Eq. 2: the transform is orthogonal.)
 *     scores[i][t] = < q_i , k_t >,   k_t the read path's reconstruction of key t (before its fp16 rounding)
 * computed as < Q (s * q_i) / max(lambda, 1e-6) , code_t * scale_t >: only the record of the keys is read.
 *   q_f16_dev      [n_q, d] fp16, 16-byte aligned, 1 <= n_q <= 32 (e.g. the query heads sharing one KV head).
 *   codes_dev      [n_keys, d/2] bytes, 16-byte aligned;  scales_dev [n_keys, d/g] fp32: the plan's record.
 *   scores_dev     [n_q, n_keys] fp32, row-major, written.
 *   workspace_dev  srft_scores_workspace_bytes(plan) bytes of device memory (about 1 MiB), 16-byte aligned;
 *                  the present kernel leaves it alone.
 * For plans with d a multiple of 64, 4-bit codes and g >= 32 (else SRFT_ERR_BAD_D / _BAD_BITS / _BAD_GROUP).
 * Enqueues one kernel on the stream.
 */
int64_t srft_scores_workspace_bytes(const srft_plan_t* plan);
int srft_kv_scores(const srft_plan_t* plan, const void* q_f16_dev, int n_q, const uint8_t* codes_dev,
                   const float* scales_dev, int64_t n_keys, float* scores_dev, void* workspace_dev,
                   void* hip_stream);

/*
 * Weighted sums of stored values, without reconstructing the values: the other half of attention over the stored
 * cache.    (Sec. 1 and Sec. 7.2: attention reads the prefix the cache holds; Eq. 1-2: the transform is linear.)
 *     out[i] = sum_t weights[i][t] * v_t,   v_t the read path's reconstruction of value t (before its fp16 rounding)
 * computed as one inverse transform per query of  sum_t weights[i][t] * code_t * scale_t : only the record is read.
 *   weights_f32_dev [n_q, n_keys] fp32 row-major, 4-byte aligned, 1 <= n_q <= 32 (e.g. softmax of srft_kv_scores).
 *   codes_dev       [n_keys, d/2] bytes, 16-byte aligned;  scales_dev [n_keys, d/g] fp32: the plan's record.
 *   out_f32_dev     [n_q, d] fp32, written.
 *   workspace_dev   srft_attend_workspace_bytes(plan) bytes of device memory (about 34 MiB at d = 128), 16-byte aligned,
 *                   overwritten; calls that may run at the same time need a workspace each.
 * n_keys >= 1.  For plans with d a multiple of 64, 4-bit codes and g >= 32 (else SRFT_ERR_BAD_D / _BAD_BITS /
 * _BAD_GROUP).  Enqueues three kernels: partial sums per workgroup (fp32, on the matrix cores), their sum in a fixed
 * order (two levels), and the inverse transform.  The result does not depend on timing.
 */
int64_t srft_attend_workspace_bytes(const srft_plan_t* plan);
int srft_kv_attend(const srft_plan_t* plan, const float* weights_f32_dev, int n_q, const uint8_t* codes_dev,
                   const float* scales_dev, int64_t n_keys, float* out_f32_dev, void* workspace_dev,
                   void* hip_stream);

/*
 * One decode step of attention over a stored cache: out = softmax(softmax_scale * q K^T) V with K and V read from
 * their records (plan_k, plan_v: same d, own signs and lambda each).    (Sec. 1; Sec. 7.2)
 * On one stream, two kernels: one pass over both records that carries scores, a running softmax and the weighted sums of
 * the values in registers, then the addition of the workgroups' sums (in a fixed order), the division and the inverse
 * transform.  q_f16_dev [n_q, d] fp16 (16-byte aligned),
 * out_f32_dev [n_q, d] fp32; workspace_dev: srft_decode_attention_workspace_bytes(plan_k, plan_v, n_q, n_keys) bytes,
 * 256-byte aligned, overwritten.  Shapes and limits as for srft_kv_scores and srft_kv_attend.
 */
int64_t srft_decode_attention_workspace_bytes(const srft_plan_t* plan_k, const srft_plan_t* plan_v, int n_q,
                                              int64_t n_keys);
int srft_kv_decode_attention(const srft_plan_t* plan_k, const srft_plan_t* plan_v, const void* q_f16_dev, int n_q,
                             const uint8_t* k_codes_dev, const float* k_scales_dev, const uint8_t* v_codes_dev,
                             const float* v_scales_dev, int64_t n_keys, float softmax_scale, float* out_f32_dev,
                             void* workspace_dev, void* hip_stream);

/*
 * srft_kv_scores for callers that cannot allocate device memory or pass a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, checks and results as
 * srft_kv_scores without workspace_dev.  Calls no hipMalloc, hipFree or other allocating routine.
 */
int srft_kv_scores_static(const srft_plan_t* plan, const void* q_f16_dev, int n_q, const uint8_t* codes_dev,
                          const float* scales_dev, int64_t n_keys, float* scores_dev, void* hip_stream);

/*
 * Cache manager: int4 store + fp16 residual window + dequantized-prefix cache.   (Sec. 7.2: the cache class,
 * items (i)-(iv), and its paragraph on the residual window: 16 tokens.)
 *
 * One cache holds n_plans (layer, K|V) plans of one shape, each with n_seq sequences (batch x kv_heads) that grow
 * in lock-step.  All device buffers belong to the caller, one per plan, in a paged layout whose page is the
 * residual window of R tokens:
 *     codes_dev[p]     [capacity/R][n_seq][R][d/2]  bytes      the int4 store ([..][d] at 8 bits)  (16-byte aligned)
 *     scales_dev[p]    [capacity/R][n_seq][R][d/g]  fp32                                  (4-byte aligned)
 *     view_f16_dev[p]  [capacity/R][n_seq][R][d]    fp16       what attention reads       (16-byte aligned)
 * Token j of sequence q is at page j / R, slot j % R.  In the view, tokens below srft_cache_quantized_tokens() hold
 * what the store decodes to (the dequantized prefix, written once when their page is flushed, never again: an
 * update costs O(1) in the prefix length); tokens from there up to srft_cache_tokens() are the residual window,
 * exact fp16 copies of what was appended.  The store holds the quantized tokens only.
 *
 * srft_cache_create   records the geometry and the pointers (host arrays of n_plans entries, copied); no HIP
 *                     calls.  capacity_tokens must be a positive multiple of residual_tokens (>= 1).
 * srft_cache_append   new_f16_dev: host array of n_plans device pointers, each [n_seq, t, d] fp16 (16-byte
 *                     aligned): t new tokens per sequence.  Enqueues a copy of the tokens into the view or, if one or
 *                     more pages became full, their quantization over all plans, out of the new tokens and of what the
 *                     window holds, and their decoding into the view, in one launch or two.  That takes addresses of
 *                     the plans' buffers and of the plans' device constants that lie a constant step apart, no more
 *                     plans than workgroups (srft_plan_set_max_workgroups), and pages and calls whose rows and 16-byte
 *                     units 32-bit numbers count; else it is a copy, a quantization and a decoding, each one launch
 *                     for every 64 plans.  Exceeding the capacity is SRFT_ERR_BAD_N (nothing is enqueued).  The result
 *                     does not depend on how the tokens are split into calls.
 * srft_cache_rebuild_view  dequantizes the whole store into the view again (for a caller that dropped or
 *                     overwrote the view); O(prefix).  The window part of the view is not touched.
 * Calls on one cache must be made from one thread at a time and enqueued on one stream (or ordered by the caller).
 */
typedef struct srft_cache srft_cache_t;
int srft_cache_create(srft_cache_t** out, const srft_plan_t* const* plans, int n_plans, int n_seq,
                      int64_t capacity_tokens, int residual_tokens, uint8_t* const* codes_dev,
                      float* const* scales_dev, void* const* view_f16_dev);
int srft_cache_destroy(srft_cache_t* cache);     /* NULL is accepted; the buffers stay the caller's */
int srft_cache_append(srft_cache_t* cache, const void* const* new_f16_dev, int t, void* hip_stream);
int srft_cache_rebuild_view(srft_cache_t* cache, void* hip_stream);
int64_t srft_cache_tokens(const srft_cache_t* cache);              /* tokens per sequence, or a negative status */
int64_t srft_cache_quantized_tokens(const srft_cache_t* cache);    /* of which in the int4 store */

/*
 * Calibration statistic for lambda: per-channel abs-max of the transform output over a batch.  (Sec. 7.1: lambda is
 * the reciprocal of that maximum; Sec. 7.2: one static calibration over whole windows.)
 *   x_f16_dev  [n_vec, d] fp16, 16-byte aligned.                                         read only
 *   amax_dev   d fp32 on the device, 4-byte aligned, all >= 0: a RUNNING maximum.  On return amax_dev[k] =
 *              max(old amax_dev[k], max over the n_vec vectors of |w_k|), w = lambda * pack(F (s * x)) with the
 *              plan's lambda.  Zero it before the first batch; call once per batch of the calibration window.
 *              With a plan created with lambda_host = NULL, w is the plain SRFT output.
 * Updated with atomic maxima: calls on the same amax_dev may overlap.
 */
int srft_kv_channel_absmax(const srft_plan_t* plan, const void* x_f16_dev, int64_t n_vec, float* amax_dev,
                           void* hip_stream);

/*
 * lambda from that statistic, on the host: lambda_k = 1 / amax_k (Sec. 7.1).  Two cases the paper does not cover:
 * a channel whose amax is below 2^-16 of the largest is treated as if it were at that floor (srft_plan_create
 * accepts max/min lambda up to 2^16), and an all-zero statistic gives lambda = 1.  amax_host: d finite floats >= 0
 * (else SRFT_ERR_BAD_LAMBDA); lambda_host: d floats, written.  No HIP calls.
 */
int srft_lambda_from_absmax(const float* amax_host, int d, float* lambda_host);

/*
 * Rotary positions on rows of heads, several tensors of the same tokens in one call (queries and keys).
 * The first `rot` channels of a row are rot / 2 pairs (a, b); with t = positions[token] * freq[pair]
 *     a' = factor (a cos t - b sin t),   b' = factor (a sin t + b cos t);   the channels from rot on are copied.
 * inverse != 0 turns by -t: with the same factor that is the gradient of the call with inverse = 0.
 *   rows        HOST array of `count` tensors (0 .. SRFT_ROTARY_MAX), each [n_tokens][n_heads][d] in in_dev and out_dev with the
 *               given strides in elements (the channels next to each other).  out_dev == in_dev with the same strides and type
 *               turns in place (with others: SRFT_ERR_BAD_N); overlapping otherwise is not allowed.  Every pointer is aligned to its element.
 *   layout      SRFT_ROTARY_HALF: pair i is channels i and i + rot / 2.  SRFT_ROTARY_PAIRS: channels 2 i and 2 i + 1.
 *   positions_dev  [n_tokens] int32;  freq_dev [rot / 2] fp64, radians per token (of a long context: whatever scaling the
 *               model takes, srft_rotary knows of none).  Angles are formed and reduced in 64 bits.
 * d even, 2 <= d <= 1024, rot even, 0 <= rot <= d, types of srft_dtype, n_tokens * n_heads < 2^31, n_heads * d < 2^31 (else SRFT_ERR_BAD_N).
 * n_tokens == 0 or count == 0 is a successful no-op.  One kernel for the tensors of one pair of types whose sizes, strides and addresses
 * let threads move 16 bytes at a time; those that take smaller accesses have one of their own.
 */
typedef enum srft_dtype { SRFT_F32 = 0, SRFT_F16 = 1, SRFT_BF16 = 2 } srft_dtype;
typedef enum srft_rotary_layout { SRFT_ROTARY_HALF = 0, SRFT_ROTARY_PAIRS = 1 } srft_rotary_layout;
enum { SRFT_ROTARY_MAX = 4 };
typedef struct srft_rotary_rows {
    const void* in_dev;
    void* out_dev;
    int64_t in_token, in_head, out_token, out_head;          /* strides in elements */
    int32_t n_heads;
    int32_t in_type, out_type;                               /* srft_dtype */
    int32_t reserved;                                        /* 0 */
} srft_rotary_rows;
int srft_rotary(const srft_rotary_rows* rows, int count, int64_t n_tokens, int d, int rot, int layout,
                const int32_t* positions_dev, const double* freq_dev, double factor, int inverse, void* hip_stream);

/*
 * RMS norms of rows of heads and their rotary positions, in one pass over several tensors of the same tokens (queries and keys).  A row
 * x of d channels becomes srft_rotary's turn of n, with
 *     n_i = x_i r w_i,   r = 1 / sqrt(mean_j x_j^2 + eps)          (all d channels; those from rot on are not turned).
 * The values are fp32 up to the output, which is rounded once.  A row's mean of squares must stay inside fp32.
 *   rows          HOST array of `count` tensors (0 .. SRFT_ROTARY_MAX): x as in srft_rotary, in place too (out_dev == in_dev with the same
 *                 strides and type); weight_dev [d] of weight_type (a srft_dtype), aligned to its element, or NULL: all 1.
 *   eps           from 1.17549435e-38 to 3.4e38 (else SRFT_ERR_BAD_N).
 * All else, sizes, refusals and launches, as in srft_rotary.
 *
 * srft_norm_rotary_backward: from dy, the gradient of the call's outputs, and its inputs,
 *     dx, the gradient of x, and dweight [d] fp32, that of the weights, summed over tokens and heads; both are written, not added to.
 *   dx has x's type.  dx_dev may be x_dev or dy_dev, with the same strides and type; overlapping otherwise is not allowed.  dweight_dev NULL: not
 *   asked for; two tensors have two of them (else SRFT_ERR_BAD_N).  n_tokens == 0 writes zeros there.
 *   workspace_dev  srft_norm_rotary_backward_workspace_bytes bytes, 16-byte aligned, overwritten (NULL where no dweight is asked for).
 * Sums are fp32, in an order that depends on sizes and alignment alone.
 */
typedef struct srft_norm_rows {
    srft_rotary_rows x;
    const void* weight_dev;
    int32_t weight_type;
    int32_t reserved;                                        /* 0 */
} srft_norm_rows;
int srft_norm_rotary(const srft_norm_rows* rows, int count, int64_t n_tokens, int d, int rot, int layout, const int32_t* positions_dev,
                     const double* freq_dev, double factor, double eps, void* hip_stream);
typedef struct srft_norm_grad_rows {
    const void *dy_dev, *x_dev;
    void* dx_dev;
    const void* weight_dev;
    float* dweight_dev;
    int64_t dy_token, dy_head, x_token, x_head, dx_token, dx_head;       /* strides in elements */
    int32_t n_heads;
    int32_t dy_type, x_type, weight_type;                    /* srft_dtype */
} srft_norm_grad_rows;
int64_t srft_norm_rotary_backward_workspace_bytes(int count, int d);
int srft_norm_rotary_backward(const srft_norm_grad_rows* rows, int count, int64_t n_tokens, int d, int rot, int layout,
                              const int32_t* positions_dev, const double* freq_dev, double factor, double eps, void* workspace_dev,
                              void* hip_stream);

/*
 * Paged cache of one layer: a pool of pages for K and one for V, shared by sequences of any length.     (Sec. 7.2, with the pages of
 * a sequence in any order.)  A page holds R = page_tokens tokens of n_heads key heads as the plans' record; the tokens behind a
 * sequence's last full page are exact fp16 in a window of R tokens, as in srft_cache, and become a page when the window is full:
 *     codes_dev   [n_pages][n_heads][R][d/2] bytes ([d] at 8 bits)      scales_dev  [n_pages][n_heads][R][d/g] fp32
 *     window_dev  [n_windows][n_heads][R][d] fp16                       (all 16-byte aligned)
 * All device buffers are the caller's.  Which pages and windows a sequence has is the caller's bookkeeping (page tables on the device,
 * read by the kernels, so that a step can be captured in a graph and replayed with other lengths).
 *
 * srft_pool_create   plan_k, plan_v: same d, group size, code width, transform and device.  page_tokens is 16, 32, 64, 128 or 256,
 *                    n_heads * page_tokens a multiple of 32, n_pages >= 0, n_windows >= 1 (else SRFT_ERR_BAD_N).  n_pages == 0 is a pool
 *                    of windows alone, for sequences shorter than a page: codes_dev and scales_dev are NULL then (else SRFT_ERR_BAD_N).
 *                    Allocates device tables (12 d^2 bytes, and a page of zeros where n_pages is 0) on the plans' GPU.  The plans
 *                    must outlive the pool.
 */
typedef struct srft_pool srft_pool_t;
typedef struct srft_pool_buffers {
    uint8_t* codes_dev;
    float* scales_dev;
    void* window_f16_dev;
} srft_pool_buffers;
int srft_pool_create(srft_pool_t** out, const srft_plan_t* plan_k, const srft_plan_t* plan_v, int n_heads, int page_tokens,
                     int64_t n_pages, int64_t n_windows, const srft_pool_buffers* k, const srft_pool_buffers* v);
int srft_pool_destroy(srft_pool_t* pool);        /* NULL is accepted; the buffers stay the caller's */

/*
 * The sequences of one call.  Sequence b brings the new tokens starts[b] .. starts[b + 1] - 1 (rows of k, v and q) and holds
 * lengths[b] tokens with them; its token j lies in page page_table[b][j / R] if that page is full, else in window
 * windows[b][1].  windows[b][0] is the window that it had before the call: where the call fills a page, windows[b][1] has to be
 * another window than windows[b][0] (no other sequence's either), else it is the same.
 * max_new and max_length bound what the device arrays hold: they size launches and workspaces.  What is beyond them is cut off;
 * a page or window number out of range names no memory: its tokens are neither read nor written, and count for nothing.
 * Each row belongs to one sequence at most.  Where starts give rows to several, calls keep to their buffers; which pages they fill and
 * which rows they answer is not defined then.
 * 0 <= n_seq <= 4096, 0 <= max_new, 0 <= max_length < 2^30, max_pages >= max_length / R (else SRFT_ERR_BAD_N).
 */
typedef struct srft_paged_seqs {
    int32_t n_seq;
    int32_t max_new;
    int64_t max_length;
    int64_t max_pages;               /* entries of a row of page_table */
    const int32_t* page_table_dev;   /* [n_seq][max_pages] */
    const int32_t* windows_dev;      /* [n_seq][2] */
    const int32_t* lengths_dev;      /* [n_seq] */
    const int32_t* starts_dev;       /* [n_seq + 1] */
} srft_paged_seqs;

/*
 * Append: the pages that the new tokens fill are quantized out of the window and the new tokens (the record of srft_kv_quantize, bit for
 * bit), the tokens behind them are copied into the window.  The result does not depend on how the tokens are split into calls.
 *   k_f16_dev, v_f16_dev   [n_new][n_heads][d] fp16, 16-byte aligned, strides in elements, multiples of 8.
 *   workspace_dev          srft_pool_append_workspace_bytes bytes, 16-byte aligned, overwritten.
 * The tokens must be finite.  Sizes are counted with 32 bits (else SRFT_ERR_BAD_N): with F = n_new / R + min(n_seq, n_new), the pages that a call can
 * fill at most, and T = n_heads * R / 32, n_new * n_heads, 32 F T and F T^2 stay below 2^31.
 */
int64_t srft_pool_append_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, int64_t n_new);
int srft_pool_append(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* k_f16_dev, const void* v_f16_dev,
                     int64_t n_new, int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* workspace_dev,
                     void* hip_stream);

/*
 * Attention of the new tokens over the cache that holds them: out = softmax(softmax_scale * q K^T) V, causal (the i-th of the n new
 * tokens of a sequence of length L sees the tokens 0 .. L - n + i), query head h reading key head h / (n_q_heads / n_heads).  K and V
 * are the read path's reconstruction before its fp16 rounding where a page is full, and the window's fp16 values behind it.  A row that
 * sees nothing is zero.  q, and the windows' tokens, must be finite.
 * Sums, maxima and scores' sums are fp32.  Sequences that bring up to 16 rows (new tokens times n_q_heads / n_heads), or 32 where max_new allows 17
 * to 32, round a weight times a scale to fp16: with the output's rounding to fp16, 3e-4 of an output's size.  Those that bring more also round the
 * transformed queries, scales, and code times scale: 1.2e-3, up to 1.5e-3 with one scale a row.
 *   q_dev, out_dev   [n_new][n_q_heads][d], both of `type` (SRFT_F16 or SRFT_BF16), 16-byte aligned, strides in elements, multiples of 8.
 *   n_q_heads        a multiple of n_heads, at most 64 n_heads.
 *   softmax_scale    finite.
 * Sizes are counted with 32 bits (else SRFT_ERR_BAD_N): with G = n_q_heads / n_heads, tiles = max_length / 32 + 2 and S = n_seq * n_heads,
 * 2 S tiles and (n_new * G / 256 + n_seq) * n_heads * max(tiles, 8) stay below 2^31 - 256, n_new * n_q_heads below 2^31 - 32 and
 * (S * R / 16 + 3 compute units + 1) * 2 d below 2^32.
 *   workspace_dev    srft_pool_attention_workspace_bytes bytes, 256-byte aligned, overwritten.  (Whatever srft_plan_set_max_workgroups is
 *                    called with before or after: the size does not depend on it.)
 */
int64_t srft_pool_attention_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, int64_t n_new, int n_q_heads);
int srft_pool_attention(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* q_dev, int type, int64_t n_new, int n_q_heads,
                        int64_t q_token, int64_t q_head, float softmax_scale, void* out_dev, int64_t out_token, int64_t out_head,
                        void* workspace_dev, void* hip_stream);

/*
 * Sliding attention: srft_pool_attention where a token sees, of the tokens up to itself, the last `recent` ones (itself among them) and the
 * sequence's first `sinks` ones.  Pages that no row of the call sees are not read: they may be another sequence's by then, and their entries in
 * the page table may hold anything.
 *   recent, sinks   recent >= 1, sinks >= 0 (else SRFT_ERR_BAD_N).  With recent + sinks >= max_length it is srft_pool_attention, in its sizes and with
 *                   its workspace too.
 *   workspace_dev   srft_pool_attention_sliding_workspace_bytes bytes (enough for any reach), 256-byte aligned, overwritten.
 * The sizes named at srft_pool_attention stay below the same bounds with tiles = max_length / 32 + 8 (else SRFT_ERR_BAD_N, of the workspace's size too).
 */
int64_t srft_pool_attention_sliding_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, int64_t n_new, int n_q_heads);
int srft_pool_attention_sliding(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* q_dev, int type, int64_t n_new, int n_q_heads,
                                int64_t q_token, int64_t q_head, float softmax_scale, int64_t recent, int64_t sinks, void* out_dev,
                                int64_t out_token, int64_t out_head, void* workspace_dev, void* hip_stream);

/*
 * Attention of sequences that begin with the same pages (samples of one prompt, conversations behind one long instruction: forks whose full
 * pages are not copied).  The outputs are srft_pool_attention's; the pages in common are read once for up to 256 rows of a key head, of whichever
 * of the group's sequences (for 16 or 32 in groups that bring no more than 48, or in calls of no more than 128).  Roundings are those named there,
 * where the rows of a group count together, as those of a sequence that brings many, if they are more than that (a step of 64 conversations with 8 rows
 * a key head each: 1.3e-3 of an output's size, where srft_pool_attention has 3e-4).
 * Group g is the sequences groups[g] .. groups[g + 1] - 1, whose first tokens[g] tokens lie in the same pages; of these, whole pages count
 * that all of the group's sequences with new tokens hold without them, and the entries of its first such sequence name them (those of the
 * others are not read).  Sequences outside of all groups are as in srft_pool_attention.  Groups are ascending: a bound below the one
 * in front of it, or past n_seq, is taken as that.
 *   prefixes        0 <= n_groups <= n_seq (else SRFT_ERR_BAD_N); without groups the pointers may be NULL.
 *   workspace_dev   srft_pool_attention_shared_workspace_bytes bytes, 256-byte aligned, overwritten.
 * With groups, tiles = max_length / 32 + 8 and N = n_seq + n_groups the sizes named at srft_pool_attention are (3 N + 8) * n_heads * tiles in the place of
 * 2 S tiles, and (2 n_new * G / 256 + N) * n_heads * max(tiles, 8); without groups the call is srft_pool_attention, in its sizes and with its workspace too.
 */
typedef struct srft_shared_prefixes {
    int32_t n_groups;
    int32_t reserved;                                        /* 0 */
    const int32_t* groups_dev;                               /* [n_groups + 1] */
    const int32_t* tokens_dev;                               /* [n_groups] */
} srft_shared_prefixes;
int64_t srft_pool_attention_shared_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, const srft_shared_prefixes* prefixes,
                                                   int64_t n_new, int n_q_heads);
int srft_pool_attention_shared(const srft_pool_t* pool, const srft_paged_seqs* seqs, const srft_shared_prefixes* prefixes, const void* q_dev, int type,
                               int64_t n_new, int n_q_heads, int64_t q_token, int64_t q_head, float softmax_scale, void* out_dev,
                               int64_t out_token, int64_t out_head, void* workspace_dev, void* hip_stream);

/*
 * Copies inside pools: page pages[i][0] to page pages[i][1] and window windows[i][0] to windows[i][1], K and V, in each of n_pools pools of
 * one geometry (the layers of a model): what a fork or a compaction needs.  Device arrays [n][2] of int32.  No destination may be
 * another destination or a source of the same call; a pair with a number out of range is skipped.  Up to 64 pools and 2^22 pairs of pages and
 * of windows each go into one launch.
 */
int srft_pool_copy(const srft_pool_t* const* pools, int n_pools, const int32_t* pages_dev, int64_t n_page_pairs,
                   const int32_t* windows_dev, int64_t n_window_pairs, void* hip_stream);

/* Plan introspection (host side, no HIP calls). */
int srft_plan_d(const srft_plan_t* plan);             /* d, or a negative status */
int srft_plan_group_size(const srft_plan_t* plan);    /* g */
int srft_plan_groups(const srft_plan_t* plan);        /* d / g: scales per vector */
int srft_plan_code_bytes(const srft_plan_t* plan);    /* code bytes per vector: d / 2 at 4 bits, d at 8 */
int srft_plan_bits(const srft_plan_t* plan);          /* 4 or 8 */
/* Which form of the transform the plan's launches run: path 0 = write, 1 = read; returns 0 = the whole matrix
 * (plain form), 1 = folded once, 2 = folded twice (the factorisations that the symmetries of Eq. 1-2 allow; the
 * record is the same in every form), or SRFT_ERR_NULL / SRFT_ERR_BAD_N. */
int srft_plan_form(const srft_plan_t* plan, int path);
int srft_plan_get_signs(const srft_plan_t* plan, int8_t* out_host /* d entries, each -1 or +1 */);

/*
 * Launch shape: both kernels are persistent (a fixed grid loops over tiles of 32 vectors).
 * max_workgroups > 0 caps the grid of this plan's launches (to leave compute units to other streams, or to
 * check that results do not depend on the grid); 0 restores the default (compute units x resident workgroups
 * per unit).  Records and reconstructions are bit-identical for every grid size.  (srft_pool_attention takes the cap of plan_k and, with
 * another grid, adds the sums of a row up in other parts: within the roundings named there.)  The library reads no environment variables.
 */
int srft_plan_set_max_workgroups(srft_plan_t* plan, int max_workgroups);

const char* srft_status_string(int status);
int srft_last_hip_error(void);    /* the hipError_t of the most recent SRFT_ERR_HIP on this thread */

#ifdef __cplusplus
}
#endif
#endif /* SRFT_KV_H */
