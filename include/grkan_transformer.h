/*
 * grkan_transformer.h - C ABI of the operators that stand around the KAT MLP in a
 * transformer block (gfx950): root-mean-square norm with the residual's addition,
 * rotary positions with several axes, cross attention to an encoder's states.
 *
 * Conventions are grkan.h's: DEVICE pointers, caller-owned memory, work enqueued on
 * `hip_stream` without synchronising, argument and launch errors as the status, no
 * allocation.  Strides are in elements; the last dimension of every tensor is
 * contiguous.  Results are bit-identical from run to run (fixed orders, no atomics).
 */
#ifndef GRKAN_TRANSFORMER_H_
#define GRKAN_TRANSFORMER_H_

#include "grkan.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Root-mean-square norm:
 *
 *     h = x + residual     (rounded to the I/O type; h = x where residual is NULL)
 *     y = h * s * weight,  s = 1 / sqrt(mean over the row of h^2 + eps)
 *
 *   x, residual  [rows, D] of io, rows x_stride / residual_stride apart; residual or NULL
 *   weight       [D] of weight_dtype: io's type or GRKAN_F32
 *   h            [rows, D] of io, contiguous; written where residual is given (else NULL).  May be x or
 *                residual itself, where that is contiguous.
 *   y            [rows, D], contiguous: of io or, with scale, in 8 bits
 *   scale        NULL, or float32 [rows]: then y is float8 (e4m3, OCP: largest value 448) and stands for
 *                y * scale, scale = (largest magnitude of the row) / 448; a row of zeros has scale 0.  A row with
 *                a NaN or an infinity, or whose squares' sum is past float32, has NaN as its scale.
 *
 * All arithmetic is float32; y is made of the rounded h (what the backward pass sees) and rounded once.
 * 1 <= D <= 16384, else GRKAN_ERR_UNSUPPORTED.  Pointers aligned to their elements.
 */
grkan_status_t grkan_rms_norm_fwd(const void *x, const void *residual, const void *weight, void *h, void *y, float *scale,
                                  int64_t rows, int32_t D, int64_t x_stride, int64_t residual_stride, float eps,
                                  grkan_dtype_t io, grkan_dtype_t weight_dtype, void *hip_stream);

/*
 * Its backward pass.  With n = h s and g = dy weight:
 *
 *     dx = s (g - n mean over the row of (g n)) (+ dh)       the gradient of x and of the residual alike
 *     dweight = sum over the rows of dy n
 *
 *   h   the sum that the forward pass kept (x where there was no residual); dy; dh the gradient that reaches h from
 *       elsewhere, or NULL: [rows, D] of io with row strides of their own
 *   dx  [rows, D] of io, contiguous (may be dy or dh where that is contiguous); dweight [D] of weight_dtype, overwritten
 *   workspace  grkan_rms_norm_bwd_workspace_bytes() bytes of scratch, 16-byte aligned, untouched until the enqueued work has
 *              finished (host-only query; 0 for sizes that are not supported)
 */
size_t grkan_rms_norm_bwd_workspace_bytes(int64_t rows, int32_t D, grkan_dtype_t io);
grkan_status_t grkan_rms_norm_bwd(const void *h, const void *dy, const void *dh, const void *weight, void *dx, void *dweight,
                                  void *workspace, size_t workspace_bytes, int64_t rows, int32_t D, int64_t h_stride,
                                  int64_t dy_stride, int64_t dh_stride, float eps, grkan_dtype_t io,
                                  grkan_dtype_t weight_dtype, void *hip_stream);

/*
 * Rotary positions with several axes: pair j of a head's channels is turned by the angle of its axis,
 *
 *     angle = positions[token][axis[j]] * frequencies[j]
 *     (a, b) -> (a cos(angle) - b sin(angle), a sin(angle) + b cos(angle))        inverse: by -angle
 *
 * where (a, b) are channels (j, pairs + j) or, interleaved, (2 j, 2 j + 1); channels from 2 pairs on are copied.  The backward
 * pass is the inverse.
 *
 * One or two tensors (queries and keys) in one launch.  Of each:
 *   x          [batch, tokens, heads, dim] of io, strides batch_stride, token_stride, head_stride
 *   out        the same shape, contiguous; may be x where x is contiguous
 *   positions  [batch, tokens, axes] of positions_dtype with strides position_batch_stride (0: the same for all) and
 *              position_token_stride
 * frequencies: DEVICE float64 [pairs], radians per step of position; axis: DEVICE int32 [pairs], each below `axes` (checked by
 * the caller: the kernel reads what it says, clamped to 0 .. axes - 1).
 * dim even, 4096 at most; heads x c x max(heads, c) below 2^32, with c = dim / 16 (float32: dim / 8), or 2, 4, 8 times that where
 * `pairs` or dim / 2 is not a multiple of 8 (float32: 4); workgroups of up to 512 / (heads x c) tokens, one at least, below 2^24, as a
 * launch has less than 2^32 threads: else GRKAN_ERR_UNSUPPORTED.
 * The angle is formed and reduced to one turn in float64, so that it is as exact at position 1,000,000 as at 1; sine and
 * cosine in float32, once for each token and pair.
 */
typedef enum { GRKAN_POSITIONS_I32 = 0, GRKAN_POSITIONS_I64 = 1, GRKAN_POSITIONS_F32 = 2 } grkan_positions_t;
typedef struct {
    const void *x;
    void *out;
    const void *positions;
    int64_t batch, tokens;
    int32_t heads;
    int64_t batch_stride, token_stride, head_stride;
    int64_t position_batch_stride, position_token_stride;
    grkan_positions_t positions_dtype;
} grkan_rotary_t;
grkan_status_t grkan_rotary(const grkan_rotary_t *tensors, int32_t count, const double *frequencies, const int32_t *axis,
                            int32_t pairs, int32_t axes, int32_t dim, int32_t interleaved, int32_t inverse, grkan_dtype_t io,
                            void *hip_stream);

/*
 * Cross attention: queries of one sequence attend to the states of another.  With head h of the queries reading head
 * h div (heads / kv_heads) of the keys and values:
 *
 *     P = softmax over the valid keys of (scale q k^T)         out = P v
 *
 *   q     [batch, queries, heads, dim] of io; k, v [batch, keys, kv_heads, dim]; strides of batch, token and head, each a
 *         multiple of 8 elements, and 16-byte aligned pointers (else GRKAN_ERR_ALIGN)
 *   key_lengths  NULL, or [batch] of int32 (int64 with key_lengths_64): the keys below it are valid (clamped to 0 .. keys)
 *   key_mask     NULL, or one byte for each key, not 0 where it is valid: byte b * mask_batch_stride + key * mask_key_stride.
 *                With both, a key is valid by both.
 *   What lies in keys and values that are not valid, infinities and NaN included, has no influence.  A query without a valid key
 *   gets zeros, and gives no gradient.
 *   out   [batch, queries, heads, dim] of io, contiguous, 16-byte aligned
 *   lse   NULL, or float32 [batch, kv_heads, queries, heads / kv_heads] (grkan_attention_lse_count() elements), for the
 *         backward pass: log2 of the sum of exp(scale q k^T) over the valid keys; an infinity where there is none
 * io: GRKAN_BF16 or GRKAN_F16; scores, their statistics and all sums are float32, the probabilities are rounded to io for
 * the product with v.
 * dim a multiple of 8 up to 128; scale finite and positive; queries x heads / kv_heads, keys and batch x kv_heads in 31 bits; token strides of
 * k and v that are not negative and below 2^24; batch x kv_heads x tiles of 64 rows (queries x heads / kv_heads) or 128 keys up to
 * 14,000,000, as a launch has less than 2^32 threads: else GRKAN_ERR_UNSUPPORTED.
 *
 * Backward: P is recomputed from lse.  dout strided as q is; dq as out, dk and dv [batch, keys, kv_heads, dim], contiguous,
 * 16-byte aligned, overwritten (with zeros for keys that are not valid).
 *
 * workspace: grkan_attention_workspace_bytes() bytes of scratch (host-only query; 0: none is needed and it may be NULL),
 * 16-byte aligned, untouched until the enqueued work has finished.
 */
typedef struct {
    const void *q, *k, *v;
    const void *key_lengths;
    const void *key_mask;
    int64_t batch, queries, keys;
    int32_t heads, kv_heads, dim, key_lengths_64;
    int64_t q_batch_stride, q_token_stride, q_head_stride;
    int64_t k_batch_stride, k_token_stride, k_head_stride;
    int64_t v_batch_stride, v_token_stride, v_head_stride;
    int64_t mask_batch_stride, mask_key_stride;
    float scale;
} grkan_attention_t;
size_t grkan_attention_lse_count(const grkan_attention_t *attention);
size_t grkan_attention_workspace_bytes(const grkan_attention_t *attention, int32_t backward);
grkan_status_t grkan_attention_fwd(const grkan_attention_t *attention, void *out, float *lse, void *workspace,
                                   size_t workspace_bytes, grkan_dtype_t io, void *hip_stream);
grkan_status_t grkan_attention_bwd(const grkan_attention_t *attention, const void *out, const float *lse, const void *dout,
                                   int64_t dout_batch_stride, int64_t dout_token_stride, int64_t dout_head_stride, void *dq,
                                   void *dk, void *dv, void *workspace, size_t workspace_bytes, grkan_dtype_t io,
                                   void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GRKAN_TRANSFORMER_H_ */
