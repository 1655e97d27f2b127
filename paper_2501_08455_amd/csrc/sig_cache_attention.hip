// Entry point of attention over a paged cache (include/sig_sequence.h): argument checks, the cut along the places, launches.
#include "sig_cache_attention.h"

#include "sig_context.h"

using namespace sig;

namespace {

constexpr int kMostDim = 256;
constexpr int kLeastBlocks = 8;      // of 32 places, that a cut leaves a workgroup

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

}  // namespace

extern "C" int sig_cache_attention(sig_ctx *ctx, const sig_cache_t *cache, const sig_queries_t *shape, const void *q, const int64_t *lengths, const int64_t *counts,
                                   void *out, void *hip_stream)
{
    if (!ctx || !shape) return SIG_ERR_INVALID;
    const sig_queries_t &s = *shape;
    if (!valid_type(s.type) || !valid_cache(cache, s.type) || s.B < 0 || s.T < 0 || s.heads < 1 || s.heads % cache->heads || s.window < 0 || s.sinks < 0 ||
        !(fabsf(s.scale) <= FLT_MAX))
        return SIG_ERR_INVALID;
    if (cache->key_dim > kMostDim || cache->value_dim > kMostDim) return SIG_ERR_UNSUPPORTED;
    if (s.B == 0 || s.T == 0) return SIG_OK;
    if (!q || !out || !lengths) return SIG_ERR_INVALID;
    const int64_t group = s.heads / cache->heads;
    if (s.T >= INT32_MAX - 1023 || s.B > INT32_MAX / s.heads || cache->page_tokens > INT32_MAX || cache->table_pages > INT32_MAX) return SIG_ERR_TOO_LARGE;
    const int64_t tiles = (s.T * group + kQueries - 1) / kQueries;
    if (tiles > INT32_MAX || s.B * cache->heads > INT32_MAX / tiles) return SIG_ERR_TOO_LARGE;
    CacheAttentionArgs A = {};
    A.cache = cache_arguments(*cache);
    A.q = q;
    for (int i = 0; i < 3; ++i) A.qs[i] = s.q_strides[i];
    A.lengths = lengths;
    A.counts = counts;
    A.out = out;
    A.B = s.B;
    A.T = s.T;
    A.heads = s.heads;
    A.group = (int)group;
    A.window = s.window;
    A.sinks = s.sinks;
    A.power = fmaxf((float)(fabs((double)s.scale) * 1.4426950408889634), FLT_MIN);      // (see sig_window.hip)
    A.negated = s.scale < 0.0f;
    A.tiles = (int)tiles;
    // Parts of the places: as many as give two workgroups a unit, of eight blocks a part at least (two for each wavefront)
    const int64_t lines = s.B * cache->heads * tiles, places = cache->table_pages * cache->page_tokens;
    const int64_t most = s.window > 0 ? least(places, least(s.window, places) + least(s.sinks, places) + kQueries) : places;
    A.splits = 1;
    if (lines < 2 * ctx->num_cu) A.splits = (int)least((2 * ctx->num_cu + lines - 1) / lines, (most + 32 * kLeastBlocks - 1) / (32 * kLeastBlocks));
    if (A.splits < 1) A.splits = 1;
    if (A.splits > kMostSplits) A.splits = kMostSplits;
    A.quotient = Quotient(cache->page_tokens);
    const hipStream_t st = (hipStream_t)hip_stream;
    Scratch scratch;
    if (A.splits > 1) {
        const int rc = scratch.get(ctx, (size_t)(lines * A.splits * kQueries * (cache->value_dim + 2)) * sizeof(float), st, &A.parts);
        if (rc != SIG_OK) return rc;
    }
    const bool narrow = cache->type == SIG_E4M3;
    const hipError_t e = s.type == SIG_F32 ? launch_cache_attention_f32(A, narrow, st)
                         : s.type == SIG_BF16 ? launch_cache_attention_bf16(A, narrow, st) : launch_cache_attention_f16(A, narrow, st);
    return e == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}
