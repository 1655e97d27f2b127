// Linear attention in chunks: how calls are cut, and what joins the segments of a sequence that different workgroups take.
#include "sig_attention_chunk.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;

// Each segment's own state -> what lies before the next one
__global__ __launch_bounds__(kThreads) void sig_attention_join_kernel(ChunkArgs G)
{
    constexpr int AHEAD = 8;      // loads in flight
    const AttentionArgs &A = G.a[blockIdx.y];
    const int64_t size = (int64_t)A.rows * A.columns, all = A.B * A.heads * size;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (at >= all) return;
    const int64_t at_head = at / size, row = at % size / A.columns, column = at % A.columns;
    const int64_t length = attention_length(A, at_head / A.heads);
    const float g = A.log_decay[at_head % A.heads];
    const Decay whole(g, (float)G.segment_tokens);
    float *states = G.states + blockIdx.y * G.states_apart + at;
    float s = A.state ? A.state[at_head * size + row * A.row_stride + column * A.column_stride] : 0.0f;
    if (A.state && A.state == A.state_out) states[(G.segments - 1) * all] = s;
    for (int first = 0; first < G.segments - 1; first += AHEAD) {
        float own[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) own[i] = first + i < G.segments - 1 ? states[(first + i) * all] : 0.0f;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (first + i >= G.segments - 1) break;
            const int64_t n = length - (first + i) * G.segment_tokens;
            if (n >= G.segment_tokens) s = whole(s) + own[i];
            else if (n > 0) s = Decay(g, (float)n)(s) + own[i];
            states[(first + i) * all] = s;
        }
    }
}

struct Cut {
    int nv, segments;      // 64 nv columns of the state a workgroup, workgroups along time
    int64_t segment_tokens;
};

// How many columns a workgroup takes and how many workgroups share a sequence, measured (us, forward; gradient):
//   bf16, 128 x 128, 128 heads     one segment of 128 columns   of 64 columns   four segments of 128 columns
//     4,096 tokens                 319; 495                     224; 523        216; 586
//     1,024 tokens                 81; 113                      61; 124         80; 188
//   f32, 128 x 128, 128 heads, 1,024 tokens   199; 352          130; 332        166; 438
// Workgroups of 128 columns, which share the operands' loads and the pairs of a chunk, where they are more than the units (float32, bound by
// its products: where they are twice as many); else of 64 where those are about one a unit; fewer than that are cut along time, which costs a
// second read of y and z, the segments' states and two more launches (8 heads, 65,536 tokens: 16, 32, 64 and 96 segments 472, 268, 231 and
// 262; 16 heads of 64 x 64, 8,192 tokens: 1, 16, 32 and 64 segments 324, 48, 43 and 51).  As many segments as fill the units with what they hold of
// such workgroups at once: two, or three of small states (61 sequences of 2,819 tokens at most, 3 heads of 64 x 33 bfloat16: 131 us cut for two,
// 98 for three), of four chunks or more.  Segments are of 128 columns where a sequence has enough of those, nearly, to fill the units, else of
// 64 (2 to 64 heads of 128 x 128 bfloat16: 300 tokens 30; 23, 1,000 tokens 47 to 58; 34 to 51, 8 heads of 8,000 62; 55; float32 300
// tokens 60 to 68; 42 to 49).
// Long sequences of less than two workgroups of 64 columns a unit are cut too, where that pays.  Whole; cut as the rule has it (us):
//   bf16, heads   200 of 64 x 64   256 of 64 x 64   256 of 96 x 64   200 of 128 x 64   100 of 128 x 128   128 of 128 x 128   140 of 128 x 128
//   1,024 tokens  49; 54           47; 55           58; 70           62; 75            59; 74             63; 84             78; 96
//   2,048         86; 81           86; 86           113; 118         115; 123          110; 106           111; 123           145; 147
//   4,096         166; 161         167; 174         223; 212         223; 220          219; 175           221; 209           283; 267
//   8,192         325; 326         334; 344         460; 416         444; 419          459; 338           448; 394           567; 487
// (4,096 tokens of 200 heads of 128 x 128, which fill the units with two segments, 298; 334, of 128 heads of 256 x 128 346; 359.)  Float32 of at most
// 64 columns only beyond one workgroup a unit, whose second round is then shared out (4,096 tokens: 200 heads of 64 x 64 317; 323, 256 of 96 x 64
// 454; 470, 280 of 64 x 64 487; 463), of more also below (100 heads of 64 x 128 317; 274).
Cut cut_of(const AttentionArgs *a, int passes, int type, int cus)
{
    const int chunk = type == SIG_BF16 ? 64 : 32;
    bool wide = false, small = true, low = true;
    for (int i = 0; i < passes; ++i) {
        wide = wide || (a[i].columns > 64 && a[i].rows <= 128);      // (registers)
        small = small && a[i].rows <= (type == SIG_BF16 ? 64 : 96);
        low = low && a[i].rows <= 128;
    }
    auto workgroups = [&](int nv) {
        int64_t n = 0;
        for (int i = 0; i < passes; ++i) n += a[i].B * a[i].heads * ((a[i].columns + 64 * nv - 1) / (64 * nv));
        return n;
    };
    Cut cut = {wide && 4 * workgroups(2) >= (type == SIG_BF16 ? 5 : 8) * cus ? 2 : 1, 1, a[0].T};
    const int64_t chunks = (a[0].T + chunk - 1) / chunk, n = workgroups(cut.nv);
    const auto filling = [&](int nv) { return (small && nv == 1 ? 3 : 2) * cus / workgroups(nv); };      // segments: that many workgroups a unit
    const bool few = 4 * n < 3 * cus, less = !few && cut.nv == 1 && n < 2 * cus;
    const bool pays = type == SIG_BF16 ? small ? chunks >= 32 : low && chunks >= 48 && (!wide || filling(2) >= 3) : small && chunks >= 48 && (wide || n > cus);
    if (few || (less && pays)) {
        if (wide && 5 * (chunks / 4) >= 4 * filling(2)) cut.nv = 2;
        int64_t segments = filling(cut.nv);
        if (segments > chunks / 4) segments = chunks / 4;
        if (segments < 1) segments = 1;
        const int64_t each = (chunks + segments - 1) / segments;
        cut.segments = (int)((chunks + each - 1) / each);
        cut.segment_tokens = each * chunk;
    }
    return cut;
}

int64_t states_of(const AttentionArgs &A, const Cut &cut) { return cut.segments > 1 ? cut.segments * A.B * A.heads * A.rows * A.columns : 0; }

// passes that one launch takes together: as many of the next ones as hold the same rows
int together(const AttentionArgs *a, int passes, int type)
{
    int n = 1;
    while (n < passes && n < kMostPasses && chunk_rows(a[n].rows, type) == chunk_rows(a[0].rows, type)) ++n;
    return n;
}

}  // namespace

namespace sig {

int64_t attention_chunk_scratch_floats(const AttentionArgs *a, int passes, int type, int cus)
{
    int64_t most = 0;
    for (int first = 0, n; first < passes; first += n) {
        n = together(a + first, passes - first, type);
        const int64_t floats = n * states_of(a[first], cut_of(a + first, n, type, cus));
        if (floats > most) most = floats;
    }
    return most;
}

hipError_t launch_attention_chunk(const AttentionArgs *a, int passes, int type, int out_type, float *scratch, int cus, hipStream_t st)
{
    const auto launch = type == SIG_BF16 ? launch_chunk_bf16 : type == SIG_F16 ? launch_chunk_f16 : launch_chunk_f32;
    const bool partial = out_type != type;
    for (int first = 0, n; first < passes; first += n) {
        n = together(a + first, passes - first, type);
        const Cut cut = cut_of(a + first, n, type, cus);
        ChunkArgs G = {{}, n, cut.segments, cut.segment_tokens, states_of(a[first], cut), scratch};
        for (int i = 0; i < n; ++i) G.a[i] = a[first + i];
        if (cut.segments > 1) {
            launch(G, cut.nv, false, partial, st);
            const int64_t values = G.a[0].B * G.a[0].heads * G.a[0].rows * G.a[0].columns;
            sig_attention_join_kernel<<<dim3((unsigned)((values + kThreads - 1) / kThreads), (unsigned)n), kThreads, 0, st>>>(G);
        }
        launch(G, cut.nv, true, partial, st);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace sig
