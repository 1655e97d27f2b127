// Linear attention in chunks: how a call is cut, and what joins the pieces of a sequence that different workgroups take.
#include "sig_attention_chunk.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;

// states[segment] from each segment's own state to what lies before it; the state behind the last one to A.state_out
__global__ __launch_bounds__(kThreads) void sig_attention_join_kernel(ChunkArgs G)
{
    const AttentionArgs &A = G.a;
    const int64_t size = (int64_t)A.rows * A.columns, all = A.B * A.heads * size;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (at >= all) return;
    const int64_t at_head = at / size, row = at % size / A.columns, column = at % A.columns;
    const int64_t place = at_head * size + row * A.row_stride + column * A.column_stride;
    const int64_t length = attention_length(A, at_head / A.heads);
    const float g = A.log_decay[at_head % A.heads];
    float s = A.state ? A.state[place] : 0.0f;
    for (int i = 0; i < G.segments; ++i) {
        int64_t n = length - i * G.segment_tokens;
        if (n > G.segment_tokens && i + 1 < G.segments) n = G.segment_tokens;
        const float own = G.states[i * all + at];
        G.states[i * all + at] = s;
        if (n > 0) s = fmaf(s, expm1f((float)n * g), s) + own;
    }
    if (A.state_out) A.state_out[place] = s;
}

struct Cut {
    int nv, segments;      // 64 nv columns of the state a workgroup, workgroups along time
    int64_t segment_tokens;
};

Cut cut_of(const AttentionArgs &A, int type, int cus)
{
    const int chunk = type == SIG_BF16 ? 64 : 32;
    Cut cut;
    cut.nv = A.columns > 64 && A.rows <= 128 ? 2 : 1;
    const int64_t workgroups = A.B * A.heads * ((A.columns + 64 * cut.nv - 1) / (64 * cut.nv)), chunks = (A.T + chunk - 1) / chunk;
    int64_t segments = workgroups >= cus ? 1 : 2 * cus / workgroups;
    if (segments > chunks / 4) segments = chunks / 4 > 1 ? chunks / 4 : 1;
    const int64_t each = (chunks + segments - 1) / segments;
    cut.segments = (int)((chunks + each - 1) / each);
    cut.segment_tokens = each * chunk;
    return cut;
}

}  // namespace

namespace sig {

int64_t attention_chunk_scratch_floats(const AttentionArgs &A, int type, int cus)
{
    const Cut cut = cut_of(A, type, cus);
    return cut.segments > 1 ? cut.segments * A.B * A.heads * A.rows * A.columns : 0;
}

hipError_t launch_attention_chunk(const AttentionArgs &A, int type, int out_type, float *scratch, int cus, hipStream_t st)
{
    const Cut cut = cut_of(A, type, cus);
    const ChunkArgs G = {A, cut.segment_tokens, cut.segments, scratch};
    const auto launch = type == SIG_BF16 ? launch_chunk_bf16 : type == SIG_F16 ? launch_chunk_f16 : launch_chunk_f32;
    const bool partial = out_type != type, exact = A.exact;
    if (cut.segments > 1) {
        launch(G, cut.nv, false, partial, exact, st);
        const int64_t values = A.B * A.heads * A.rows * A.columns;
        sig_attention_join_kernel<<<(unsigned)((values + kThreads - 1) / kThreads), kThreads, 0, st>>>(G);
    }
    launch(G, cut.nv, true, partial, exact, st);
    return hipGetLastError();
}

}  // namespace sig
