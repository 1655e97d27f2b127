/*
 * sig_sequence.h -- C ABI of libsig's sequence-model operators: what stands behind the every-prefix signature in a model
 * that is trained on it.  Layer norm of rows, rotary positions, and linear attention with a decay for each head, each
 * with its gradient.  The conventions are those of sig.h: DEVICE pointers, a hipStream_t passed as void*, no
 * synchronisation, a status code for every failure, context scratch as described there (each entry point says what it
 * keeps there), deterministic results (no atomics, fixed summation order).
 *
 * Values are float32, bfloat16 or float16 in memory (enum sig_type).  Sums, statistics and states are in float32 or more; each
 * output is rounded once.  Arithmetic is float32's too, but for one thing: attention of bfloat16 over more than four tokens (more than two in
 * the gradient) multiplies with the state, and with the products of queries and keys, rounded to 16 digits, for outputs that
 * have 8.  The state itself, and so state_out and grad_initial, keeps float32's.  Pointers are aligned to their type, no more is asked for.
 */
#ifndef SIG_SEQUENCE_H
#define SIG_SEQUENCE_H

#include <stdint.h>

#include "sig.h"

#ifdef __cplusplus
extern "C" {
#endif

enum sig_type { SIG_F32 = 0, SIG_BF16 = 1, SIG_F16 = 2 };

/*
 * Layer norm of each row:  h = (x - mean x) / sqrt(mean (x - mean x)^2 + eps),  y = h * weight + bias.
 *   x            DEVICE, [rows][width] of `type`, rows x_stride values apart (negative and zero strides are fine), a row contiguous
 *   weight, bias DEVICE, [width] of `weight_type` (SIG_F32 or `type`), each may be NULL (1 and 0)
 *   y            DEVICE, [rows][width] of `type`, contiguous; must not overlap the inputs
 *   stats        DEVICE, float32 [rows][2], what sig_layer_norm_backward needs (mean, 1 / sqrt(...)); may be NULL
 * rows == 0 returns SIG_OK and launches nothing; width < 1, rows < 0 or a NaN or negative eps are SIG_ERR_INVALID; rows of more than 16,384
 * values that are 2^24 pieces of 8,192 or more are SIG_ERR_TOO_LARGE.
 * NaN and Inf spoil their own row only.  Statistics have float32's range: a row whose squared deviations add up to more than 3e38 has a variance of
 * infinity, and h = 0.  Any width: rows of up to 16,384 values stay on chip between their
 * statistics and their output, longer ones are read twice and cut across workgroups (context scratch of about 2 floats for
 * every 8,192 values).
 */
int sig_layer_norm(sig_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int64_t width, int type, const void *weight,
                   const void *bias, int weight_type, double eps, void *y, float *stats, void *hip_stream);

/*
 * Gradient of sig_layer_norm.  With g = grad_out * weight and means over a row:
 *   grad_x = (g - mean g - h mean(g h)) / sqrt(...),  grad_weight = sum over rows of grad_out * h,  grad_bias = sum over rows of grad_out
 *   x, weight, stats   as sig_layer_norm read and wrote them
 *   grad_out           DEVICE, [rows][width] of `type`, rows grad_stride values apart
 *   grad_x             DEVICE, [rows][width] of `type`, contiguous; may be NULL
 *   grad_weight, grad_bias  DEVICE, [width] of `weight_type`; each may be NULL.  rows == 0 leaves zeros in them
 * Context scratch for partial sums of the weights' gradients: 2 * width floats for each of some workgroups.
 */
int sig_layer_norm_backward(sig_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int64_t width, int type, const void *weight,
                            int weight_type, const float *stats, const void *grad_out, int64_t grad_stride, void *grad_x,
                            void *grad_weight, void *grad_bias, void *hip_stream);

enum sig_position { SIG_POSITION_I32 = 0, SIG_POSITION_I64 = 1, SIG_POSITION_F32 = 2, SIG_POSITION_F64 = 3 };

/*
 * Rotary positions of a [B][T][heads][dim] array.  Of the first `turned` components of each head the pair (a, b) number i,
 * components (i, i + turned / 2), or (2 i, 2 i + 1) with `interleaved`, becomes
 *   scale * (a cos t - b sin t,  a sin t + b cos t),   t = position * frequencies[i];
 * the other components are copied.  inverse != 0 turns by -t: with the same scale, the gradient.
 *   x, y         DEVICE, `type`; strides in values between batches, tokens and heads (NULL: contiguous); the last axis is
 *                contiguous.  y may be x itself (the same pointer and strides), and must not overlap it otherwise
 *   positions    DEVICE, of `position_type`, position_strides[2] values apart between batches and tokens (0: shared);
 *                whole positions, or times (irregular series)
 *   frequencies  DEVICE, float64 [turned / 2], radians a position
 * The angle is reduced in 64 bits, so that far positions keep their digits.  turned is even, 0 <= turned <= dim; more than 4,096 turned
 * components are SIG_ERR_UNSUPPORTED, 2^31 tokens (B * T) or more, or so many values of a token, SIG_ERR_TOO_LARGE.
 */
int sig_rotary(sig_ctx *ctx, const void *x, const int64_t *x_strides, void *y, const int64_t *y_strides, int type, int64_t B, int64_t T,
               int64_t heads, int64_t dim, int64_t turned, const void *positions, int position_type, const int64_t *position_strides,
               const double *frequencies, int interleaved, double scale, int inverse, void *hip_stream);

/*
 * Linear attention with a decay for each head.  With l = exp(log_decay[head]):
 *   S_t = l S_{t-1} + k_t (x) v_t,   o_t = scale * q_t S_t
 * where S is key_dim x value_dim, one for each batch element and head, and S_{-1} the initial state.
 *   q            DEVICE, [B][T][heads][key_dim] of `type`
 *   k, v         DEVICE, [B][T][shared_heads][key_dim or value_dim]; head h reads shared head h / (heads / shared_heads)
 *                strides in values between batches, tokens and heads; the last axis is contiguous
 *   log_decay    DEVICE, float32 [heads]; 0 forgets nothing, -inf everything
 *   state        DEVICE, float32 [B][heads][key_dim][value_dim]: S_{-1}; NULL: zeros
 *   lengths      DEVICE, int64 [B], tokens of each batch element (taken into 0 ... T); NULL: T.  The tokens behind them are
 *                not read, give zeros, and leave the state alone
 *   out          DEVICE, [B][T][heads][value_dim] of `type`, contiguous
 *   state_out    DEVICE, as `state` (and may be the same array): the state behind the last token; may be NULL
 * T == 1 is the form for single tokens.  Dimensions 1 ... 256 (larger ones are SIG_ERR_UNSUPPORTED); T == 0 copies the state; B == 0 does
 * nothing.  2^24 heads or more, or 2^31 states, are SIG_ERR_TOO_LARGE; what one launch cannot hold is taken in slices of the batch.
 * Context scratch where few heads' long sequences are cut along time: a state for each segment, of at most three workgroups for each
 * compute unit; else none.
 */
typedef struct sig_attention_t {
    int64_t B, T;
    int32_t heads, shared_heads, key_dim, value_dim;
    int32_t type;
    float scale;
    int64_t q_strides[3], k_strides[3], v_strides[3];
} sig_attention_t;

int sig_linear_attention(sig_ctx *ctx, const sig_attention_t *shape, const void *q, const void *k, const void *v, const float *log_decay,
                         const float *state, const int64_t *lengths, void *out, float *state_out, void *hip_stream);

/*
 * Gradient of sig_linear_attention with respect to q, k, v and the initial state (log_decay is a constant of the model).
 *   grad_out     DEVICE, [B][T][heads][value_dim] of `type`, contiguous; what stands behind the lengths is not read
 *   grad_state   DEVICE, float32, gradient with respect to state_out; NULL: zeros
 *   grad_q, grad_k, grad_v   DEVICE, shapes of q, k and v, contiguous, `type`; zeros behind the lengths; the gradient of a
 *                shared head is the sum over the heads that read it
 *   grad_initial DEVICE, float32, gradient with respect to `state`; may be NULL; overlaps no other argument
 * Context scratch as above, for up to three passes at once; and where heads share keys and values, B * T * heads * (key_dim + value_dim)
 * floats for what is added up (a batch for which that exceeds 8 GiB is taken in slices that share the scratch).
 */
int sig_linear_attention_backward(sig_ctx *ctx, const sig_attention_t *shape, const void *q, const void *k, const void *v,
                                  const float *log_decay, const float *state, const int64_t *lengths, const void *grad_out,
                                  const float *grad_state, void *grad_q, void *grad_k, void *grad_v, float *grad_initial, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SIG_SEQUENCE_H */
