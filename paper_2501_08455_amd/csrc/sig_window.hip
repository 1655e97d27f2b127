// Entry points of softmax attention with a sliding window (include/sig_sequence.h): argument checks and launches.
#include "sig_window.h"

#include "sig_context.h"

using namespace sig;

namespace {

constexpr int kMostDim = 256;
constexpr double kLog2E = 1.4426950408889634;
constexpr int kMostParts = 64;      // of a tile's queries
constexpr int kMostCut = 16;        // workgroups a unit that the first tokens' tiles are cut into

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

int check(const sig_ctx *ctx, const sig_window_t *s)
{
    if (!ctx || !s || s->B < 0 || s->T < 0 || s->heads < 1 || s->shared_heads < 1 || s->heads % s->shared_heads || s->key_dim < 1 || s->value_dim < 1 ||
        s->window < 0 || s->sinks < 0 || !valid_type(s->type) || !(fabsf(s->scale) <= FLT_MAX))
        return SIG_ERR_INVALID;
    if (s->key_dim > kMostDim || s->value_dim > kMostDim) return SIG_ERR_UNSUPPORTED;
    // (2^33 workgroups of 64 tokens or more; a grid of them holds 2^23 - 1 by 2^16 - 1)
    if (s->T >= INT32_MAX - 1023 || s->B > INT32_MAX / s->heads || (s->T > 0 && s->B * s->heads > ((int64_t)1 << 39) / (s->T + 127))) return SIG_ERR_TOO_LARGE;
    // (tiles of 16 queries or more, of all heads that share a key, are counted in 32 bits)
    if ((s->T + 15) / 16 * (s->heads / s->shared_heads) >= INT32_MAX / 2) return SIG_ERR_TOO_LARGE;
    return SIG_OK;
}

WindowArgs arguments(const sig_window_t &s, const void *q, const void *k, const void *v, const int64_t *lengths)
{
    WindowArgs A = {};
    A.q = q;
    A.k = k;
    A.v = v;
    for (int i = 0; i < 3; ++i) {
        A.qs[i] = s.q_strides[i];
        A.ks[i] = s.k_strides[i];
        A.vs[i] = s.v_strides[i];
    }
    A.lengths = lengths;
    A.B = s.B;
    A.T = (int)s.T;
    A.heads = s.heads;
    A.group = s.heads / s.shared_heads;
    A.K = s.key_dim;
    A.V = s.value_dim;
    A.window = (int)(s.window == 0 || s.window > s.T ? s.T : s.window);
    A.sinks = (int)(s.sinks > s.T ? s.T : s.sinks);
    A.scale = s.scale;
    // (a scale of 0 is taken as the smallest one, so that the scores of what is hidden stay minus infinity)
    A.power = fmaxf((float)(fabs((double)s.scale) * kLog2E), FLT_MIN);
    A.negated = s.scale < 0.0f;
    const int rows = window_rows(s.type, A.K, A.V);
    A.tiles = (A.T + rows - 1) / rows;
    A.splits = 1;
    return A;
}

// Queries that are fewer than two workgroups a unit are cut along their keys into as many pieces as give two, of 512 keys or more, or of 256 where half of the units would have
// nothing to do.  Forward, forward and gradient, us, without and with: 1 x 1,024 tokens, 1 head of 128 bfloat16 32, 102 and 18, 75; 1 x 2,048, 8 heads (2 shared) of 128 58, 207 and 37, 140;
// 1 x 16,384, 1 head of 128 410, 1,226 and 132, 538; 1 x 1,200, 2 heads of 64 float32 81, 200 and 31, 95; 1 x 2,937, 2 heads of 256 float32 522, 1,400 and 136, 542.  (8 x 512, 8 heads
// of 128 bfloat16, 256 workgroups, in pieces of 256: 142 and 155 with the gradient)
int splits_of(const sig_ctx *ctx, const WindowArgs &A, int rows)
{
    const int64_t blocks = A.B * A.heads * A.tiles, keys = A.window < A.T ? least(A.T, (int64_t)A.window + rows + A.sinks) : A.T;
    if (blocks >= 2 * ctx->num_cu) return 1;
    const int64_t splits = least((2 * ctx->num_cu + blocks - 1) / blocks, keys / (blocks < ctx->num_cu ? 256 : 512));
    return splits < 1 ? 1 : (int)splits;
}

hipError_t launch(const WindowArgs &A, int type, WindowPass pass, hipStream_t st)
{
    return type == SIG_F32 ? launch_window_f32(A, pass, st) : type == SIG_BF16 ? launch_window_bf16(A, pass, st) : launch_window_f16(A, pass, st);
}

}  // namespace

extern "C" {

int sig_window_attention(sig_ctx *ctx, const sig_window_t *shape, const void *q, const void *k, const void *v, const int64_t *lengths, void *out,
                         float *stats, void *rest, void *hip_stream)
{
    const int rc = check(ctx, shape);
    if (rc != SIG_OK) return rc;
    if (shape->B == 0 || shape->T == 0) return SIG_OK;
    if (!q || !k || !v || !out || (stats && !rest && shape->type != SIG_F32)) return SIG_ERR_INVALID;
    WindowArgs A = arguments(*shape, q, k, v, lengths);
    A.out = out;
    A.stats = (float2 *)stats;
    A.rest = stats ? (Rest *)rest : nullptr;
    A.splits = splits_of(ctx, A, window_rows(shape->type, A.K, A.V));
    Scratch scratch;
    if (A.splits > 1) {
        const int got = scratch.get(ctx, (size_t)(A.B * A.heads * A.splits * A.T * (A.V + 2)) * sizeof(float), (hipStream_t)hip_stream, &A.pieces);
        if (got != SIG_OK) return got;
    }
    return launch(A, shape->type, WINDOW_FORWARD, (hipStream_t)hip_stream) == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}

int sig_window_attention_backward(sig_ctx *ctx, const sig_window_t *shape, const void *q, const void *k, const void *v, const int64_t *lengths,
                                  const void *out, const float *stats, const void *rest, const void *grad_out, void *grad_q, void *grad_k, void *grad_v, void *hip_stream)
{
    int rc = check(ctx, shape);
    if (rc != SIG_OK) return rc;
    if (shape->B == 0 || shape->T == 0) return SIG_OK;
    if (!q || !k || !v || !out || !stats || !grad_out || !grad_q || !grad_k || !grad_v || (!rest && shape->type != SIG_F32)) return SIG_ERR_INVALID;
    const hipStream_t st = (hipStream_t)hip_stream;
    WindowArgs A = arguments(*shape, q, k, v, lengths);
    A.out = (void *)out;
    A.stats = (float2 *)stats;
    A.rest = (Rest *)rest;
    A.grad_out = grad_out;
    A.grad_q = grad_q;
    A.grad_k = grad_k;
    A.grad_v = grad_v;
    // The first tokens' tiles are cut where they have more than twice the queries of the others, unless they are so many that they balance by themselves and the parts'
    // sums would take much memory; else all tiles, where they are fewer than two a unit, into as many parts as give two, of 128 queries or more
    // (four: 2 x 1,024 tokens, 32 heads (8 shared) of 64 bfloat16 149 instead of 136 us, 1 x 8,192, 8 heads (2 shared) of 128, window 1,024, 301 instead of 287)
    const int rows = window_rows(shape->type, A.K, A.V);
    const int64_t usual = 2 * ((int64_t)A.window + rows), deltas = A.B * A.heads * A.T, lines = A.B * shape->shared_heads, all = lines * A.tiles;
    A.parts = 1;
    if (A.sinks > 0 && A.T > usual) {
        const int64_t tiles = (A.sinks + rows - 1) / rows;
        A.parts = (int)least(least(1 + (A.T + usual - 1) / usual, kMostParts), kMostCut * (int64_t)ctx->num_cu / (lines * tiles));
        if (A.parts < 2) A.parts = 1;
        if (A.parts > 1) {
            A.cut = (int)tiles;
            A.joined = A.sinks;
        }
    } else if (all < 2 * ctx->num_cu) {
        A.parts = (int)least((2 * ctx->num_cu + all - 1) / all, least(kMostParts, (least(A.T, (int64_t)A.window + rows) * A.group + 127) / 128));
        if (A.parts > 1) {
            A.cut = A.tiles;
            A.joined = A.T;
            A.even = 1;
        }
    }
    const int64_t joined = A.cut * A.parts * (int64_t)rows * (A.K + A.V) * lines;
    A.splits = splits_of(ctx, A, rows);
    const int64_t pieces = A.splits > 1 ? A.B * A.heads * A.splits * A.T * A.K : 0;
    Scratch scratch;
    rc = scratch.get(ctx, (size_t)(deltas + (joined > pieces ? joined : pieces)) * sizeof(float), st, &A.delta);
    if (rc != SIG_OK) return rc;
    A.sums = A.pieces = A.delta + deltas;      // (the pieces are joined before the keys' sums begin)
    hipError_t e = launch(A, shape->type, WINDOW_QUERY_GRADIENT, st);
    if (e == hipSuccess) e = launch(A, shape->type, WINDOW_KEY_GRADIENT, st);
    return e == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}

}  // extern "C"
