/*
 * sig_sequence.h -- C ABI of libsig's sequence-model operators: what stands behind the every-prefix signature in a model
 * that is trained on it.  Layer norm of rows, rotary positions, linear attention with a decay for each head, and softmax attention
 * with a sliding window, each with its gradient; and the paged cache that the latter is served from.  The conventions are those of sig.h: DEVICE pointers, a hipStream_t passed as void*, no
 * synchronisation, a status code for every failure, context scratch as described there (each entry point says what it
 * keeps there), deterministic results (no atomics, fixed summation order).
 *
 * Values are float32, bfloat16 or float16 in memory (enum sig_type).  Sums, statistics and states are in float32 or more; each
 * output is rounded once.  Arithmetic is float32's too, but for one thing: attention of bfloat16 over more than four tokens (more than two in
 * the gradient) multiplies with the state, and with the products of queries and keys, rounded to 16 digits, for outputs that
 * have 8.  The state itself, and so state_out and grad_initial, keeps float32's.  (Softmax attention rounds its probabilities: see there.)  Pointers are aligned to their type, no more is asked for.
 */
#ifndef SIG_SEQUENCE_H
#define SIG_SEQUENCE_H

#include <stdint.h>

#include "sig.h"

#ifdef __cplusplus
extern "C" {
#endif

enum sig_type { SIG_F32 = 0, SIG_BF16 = 1, SIG_F16 = 2, SIG_E4M3 = 3 /* of a cache's pages only */ };

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

/*
 * Softmax attention with a sliding window and first tokens that stay visible.  Token t of a sequence sees token s <= t if t - s < window
 * (window == 0: any) or s < sinks.  With z_ts = scale * q_t . k_s over what t sees:
 *   o_t = sum_s exp(z_ts) v_s / sum_s exp(z_ts)
 *   q            DEVICE, [B][T][heads][key_dim] of `type`
 *   k, v         DEVICE, [B][T][shared_heads][key_dim or value_dim]; head h reads shared head h / (heads / shared_heads)
 *                strides in values between batches, tokens and heads; the last axis is contiguous
 *   lengths      DEVICE, int64 [B], tokens of each sequence (taken into 0 ... T); NULL: T.  The tokens behind them are not read and
 *                give zeros
 *   out          DEVICE, [B][T][heads][value_dim] of `type`, contiguous
 *   stats        DEVICE, float32 [B][heads][T][2], what sig_window_attention_backward needs (a base at or near the largest z, as a power of
 *                two, and one over the sum of exp(z - base)); may be NULL.  Nothing is written for the tokens behind the lengths
 *   rest         DEVICE, a byte for each value of out, which the backward pass needs too: what out's rounding to 16 bits left (8 bits, 5 of exponent,
 *                times 2^14).  Not used, and may be NULL, with float32 and where stats is NULL
 * 16-bit operands are multiplied as they are, and the probabilities (before they are divided by their sum) rounded to that type for their product
 * with v; sums are float32's.  What a token does not see may be anything, NaN and infinities too; what is not finite spoils the tokens that see it.
 * Dimensions 1 ... 256 (larger ones are SIG_ERR_UNSUPPORTED); a scale that is not finite is SIG_ERR_INVALID; 2^31 - 1024 tokens or more, 2^31 heads
 * (B * heads) or more, 2^39 tokens of heads, or 2^30 groups of 16 tokens in the heads that
 * share one, SIG_ERR_TOO_LARGE.  B == 0 and T == 0 do nothing.  Context scratch where queries are few and see many keys, and are cut along them: value_dim + 2 floats for
 * each query and piece, of fewer than four workgroups' pieces (64 or 128 queries each) for each compute unit.
 */
typedef struct sig_window_t {
    int64_t B, T;
    int32_t heads, shared_heads, key_dim, value_dim;
    int32_t type;
    float scale;
    int64_t window, sinks;
    int64_t q_strides[3], k_strides[3], v_strides[3];
} sig_window_t;

int sig_window_attention(sig_ctx *ctx, const sig_window_t *shape, const void *q, const void *k, const void *v, const int64_t *lengths, void *out,
                         float *stats, void *rest, void *hip_stream);

/*
 * Gradient of sig_window_attention with respect to q, k and v.
 *   out, stats, rest   as sig_window_attention wrote them
 *   grad_out     DEVICE, [B][T][heads][value_dim] of `type`, contiguous; what stands behind the lengths is not read
 *   grad_q, grad_k, grad_v   DEVICE, shapes of q, k and v, contiguous, `type`; zeros behind the lengths; the gradient of a
 *                shared head is the sum over the heads that read it
 * Context scratch of B * heads * T floats; beside them the larger of key_dim floats for each query and piece (see above), and, where sequences are much longer than the window, for the sinks' gradients in up to 64 parts (16 of 64 or 128 keys for each
 * compute unit at most), or where keys are few, for all of them (fewer than four for each unit): key_dim + value_dim floats for each key and part.
 */
int sig_window_attention_backward(sig_ctx *ctx, const sig_window_t *shape, const void *q, const void *k, const void *v, const int64_t *lengths,
                                  const void *out, const float *stats, const void *rest, const void *grad_out, void *grad_q, void *grad_k, void *grad_v, void *hip_stream);

/*
 * A paged cache of keys and values.  The place p of a sequence b is slot p % page_tokens of page table[b][p / page_tokens], for all heads.
 *   keys, values DEVICE, [pages][heads][page_tokens][key_dim or value_dim] of `type`; strides in values between pages, heads and slots;
 *                the last axis is contiguous, pages do not overlap
 *   key_scales, value_scales   DEVICE, float32 [pages][heads], contiguous, for pages of SIG_E4M3 (8 bits: 4 of exponent, 3 of fraction, the largest
 *                value 448): a value stands for itself times its page's and head's scale.  NULL for the other types
 *   table        DEVICE, int32 [sequences][table_pages], rows table_stride apart
 * Places behind the table's end, and places whose page is not one of 0 ... pages - 1, do not exist: nothing is written there and nothing seen.  So
 * pages that a window has left may go to other sequences.  Calls that only read may share pages; a page that one call writes to twice, because
 * two sequences or two entries of a table name it, holds what either wrote, slot by slot (in 8 bits: with either's scale).
 */
typedef struct sig_cache_t {
    int64_t pages, page_tokens;
    int32_t heads, key_dim, value_dim;
    int32_t type;
    void *keys, *values;
    float *key_scales, *value_scales;
    int64_t key_strides[3], value_strides[3];
    const int32_t *table;
    int64_t table_pages, table_stride;
} sig_cache_t;

/*
 * Keys and values of new tokens into a cache: token t of sequence b, which holds lengths[b], goes to place lengths[b] + t.  Keys are turned on the way
 * as sig_rotary does it, and so are the tokens' queries, into an array of their own.
 * The cache's keys, values and scales lie apart from one another and from all that is read.
 *   k, v         DEVICE, [B][T][cache heads][key_dim or value_dim] of `type`; strides as everywhere
 *   q, q_out     DEVICE, [B][T][heads][key_dim] of `type`, q_out contiguous and apart from q; both NULL where heads == 0
 *   lengths      DEVICE, int64 [B] (negative ones are taken as 0)
 *   counts       DEVICE, int64 [B], new tokens of each sequence (taken into 0 ... T); NULL: T.  Those behind them are not read; their queries
 *                give zeros
 *   positions    DEVICE, of `position_type`, position_strides[2] values apart between sequences and tokens; NULL: the places
 *   frequencies  DEVICE, float64 [turned / 2]; turned, interleaved, scale: see sig_rotary.  turned == 0 leaves keys as they are
 * The cache's type is `type`, or SIG_E4M3.  Then a page's scale is the smallest power of two (2^-126 or more) that is at least the largest
 * magnitude / 448 of what it holds of a head (1 for zeros), and never less than it was while the page keeps earlier tokens: a page
 * whose slot 0 is written by the call keeps none, what another one holds is rounded anew when its scale grows (which changes only values below 2^-6 of
 * the new scale).  Values are rounded once, from float32; what is not finite is NaN there and counts as 0.
 * Limits of sig_rotary for turned; 2^31 tokens (B * T) or more, or heads or values of a token, SIG_ERR_TOO_LARGE.  No context scratch.
 */
typedef struct sig_append_t {
    int64_t B, T;
    int32_t heads, type;
    int64_t q_strides[3], k_strides[3], v_strides[3];
    const void *positions;
    int32_t position_type, interleaved;
    int64_t position_strides[2];
    const double *frequencies;
    int64_t turned;
    double scale;
} sig_append_t;

int sig_cache_append(sig_ctx *ctx, const sig_cache_t *cache, const sig_append_t *shape, const void *q, const void *k, const void *v,
                     const int64_t *lengths, const int64_t *counts, void *q_out, void *hip_stream);

/*
 * Softmax attention of the last tokens of each sequence over a cache: query t of sequence b stands at place lengths[b] - counts[b] + t and sees what
 * sig_window_attention's token there sees.  T == 1 is the form for single tokens.
 *   q            DEVICE, [B][T][heads][key_dim] of `type`; head h reads the cache's head h / (heads / cache heads)
 *   lengths      DEVICE, int64 [B]: what each sequence holds, these tokens included (places behind the table's end do not exist)
 *   counts       DEVICE, int64 [B], queries of each sequence (taken into 0 ... T); NULL: T.  Those behind them are not read and give zeros
 *   out          DEVICE, [B][T][heads][value_dim] of `type`, contiguous.  A query that sees nothing gives zeros
 * The cache's type is `type`, or SIG_E4M3.  For their product with the values probabilities of 16-bit calls keep 16 digits, over float16 pages 22 (those below e^-12 of the
 * largest: steps of 2^-39 of it, 2^-24 where scores reach 2^20); of float32 calls 24.  Sums are float32's.
 * Limits of sig_window_attention, and 2^31 - 1024 places at most; more than 2^31 groups of 16 queries are SIG_ERR_TOO_LARGE.  Context scratch where sequences are
 * cut along their places because there are few: (value_dim + 2) floats for each query and part, of fewer than four workgroups' parts (16 queries each) for each compute unit.
 */
typedef struct sig_queries_t {
    int64_t B, T;
    int32_t heads, type;
    float scale;
    int64_t window, sinks;
    int64_t q_strides[3];
} sig_queries_t;

int sig_cache_attention(sig_ctx *ctx, const sig_cache_t *cache, const sig_queries_t *shape, const void *q, const int64_t *lengths, const int64_t *counts,
                        void *out, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SIG_SEQUENCE_H */
