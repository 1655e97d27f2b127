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
    // (a grid of 2^24 x 2^15 workgroups of 64 tokens or more)
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
    return A;
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
    // sums would take much memory; else all tiles, where they are fewer than two a unit, into as many parts as give four, of 128 queries or more
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
        A.parts = (int)least((4 * ctx->num_cu + all - 1) / all, least(kMostParts, (least(A.T, (int64_t)A.window + rows) * A.group + 127) / 128));
        if (A.parts > 1) {
            A.cut = A.tiles;
            A.joined = A.T;
            A.even = 1;
        }
    }
    const int64_t joined = A.cut * A.parts * (int64_t)rows * (A.K + A.V) * lines;
    Scratch scratch;
    rc = scratch.get(ctx, (size_t)(deltas + joined) * sizeof(float), st, &A.delta);
    if (rc != SIG_OK) return rc;
    A.sums = A.delta + deltas;
    hipError_t e = launch(A, shape->type, WINDOW_QUERY_GRADIENT, st);
    if (e == hipSuccess) e = launch(A, shape->type, WINDOW_KEY_GRADIENT, st);
    return e == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}

}  // extern "C"
