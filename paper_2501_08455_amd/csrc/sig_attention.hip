// Entry points of linear attention (include/sig_sequence.h): argument checks, the passes of the gradient, and the sum
// over heads that share keys and values.
#include <type_traits>

#include "sig_attention.h"
#include "sig_context.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;
constexpr int kMostDim = 256;
constexpr int64_t kMostParts = (int64_t)8 << 30;                            // bytes of scratch for shared heads' gradients
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 32) / kThreads - 1;      // along an axis: a launch holds fewer than 2^32 threads there

// out[token][shared head][.] = sum over the heads of a shared head of part[token][head][.], in their order.  `lanes` threads (a power
// of two) take a shared head's values, N each, up to four heads' loads at once.
template <typename T, int N>
__global__ __launch_bounds__(kThreads) void sig_attention_share_kernel(const float *part, T *out, int64_t rows, int group, int dim, int lanes)
{
    const int at = threadIdx.x % lanes * N, apart = kThreads / lanes;
    if (at >= dim) return;
    for (int64_t row = (int64_t)blockIdx.x * apart + threadIdx.x / lanes; row < rows; row += (int64_t)gridDim.x * apart) {
        const float *p = part + row * group * dim + at;
        float sum[N] = {};
#pragma unroll 4
        for (int h = 0; h < group; ++h) {
            const Pack<float, N> values = load_pack<float, N>(p + (int64_t)h * dim);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += values.v[j];
        }
        Pack<T, N> result;
#pragma unroll
        for (int j = 0; j < N; ++j) result.v[j] = from_float<T>(sum[j]);
        store_pack(out + row * dim + at, result);
    }
}

int check(const sig_ctx *ctx, const sig_attention_t *s)
{
    if (!ctx || !s || s->B < 0 || s->T < 0 || s->heads < 1 || s->shared_heads < 1 || s->heads % s->shared_heads || s->key_dim < 1 ||
        s->value_dim < 1 || !valid_type(s->type))
        return SIG_ERR_INVALID;
    if (s->key_dim > kMostDim || s->value_dim > kMostDim) return SIG_ERR_UNSUPPORTED;
    if (s->heads > kMostWorkgroups || s->B > INT32_MAX / s->heads || (s->T > 0 && s->B * s->heads > INT64_MAX / (8 * kMostDim) / s->T)) return SIG_ERR_TOO_LARGE;
    return SIG_OK;
}

void contiguous(int64_t *strides, const sig_attention_t &s, int64_t heads, int64_t dim)
{
    strides[0] = s.T * heads * dim;
    strides[1] = heads * dim;
    strides[2] = dim;
}

void operand(const void **p, int64_t *strides, int *group, const void *values, const int64_t *from, int shared)
{
    *p = values;
    *group = shared;
    for (int i = 0; i < 3; ++i) strides[i] = from[i];
}

AttentionArgs pass(const sig_attention_t &s, const float *log_decay, const int64_t *lengths, int rows, int columns)
{
    AttentionArgs A = {};
    A.log_decay = log_decay;
    A.lengths = lengths;
    A.B = s.B;
    A.T = s.T;
    A.heads = s.heads;
    A.rows = rows;
    A.columns = columns;
    A.out_scale = A.update_scale = 1.0f;
    return A;
}

// Up to this many tokens go one after the other: a chunk's products cost as much for one token as for all of it.  Measured (us, token by
// token; as a chunk):
//   forward, tokens                            2           4           8            16
//   bf16, 128 sequences, 16 heads of 64 x 64   9; 16       14; 16      22; 16       38; 16
//   bf16, 64 sequences, 16 heads of 128 x 128  12; 19      20; 19      36; 19       67; 19
//   f32, 128 sequences, 4 heads of 64 x 64     5.4; 9.7    7.7; 9.6    12.6; 9.8    22.5; 10.0
// The gradient's passes are a launch each token by token, and one in chunks: 64 x 64 as above 27; 40 with two tokens, 39; 40 with four, 128 x 128
// 36; 49 and 59; 50.
constexpr int kRecurrentTokens = 4, kRecurrentGradientTokens = 2;

bool by_token(const AttentionArgs *a, bool gradient) { return a[0].T <= (gradient ? kRecurrentGradientTokens : kRecurrentTokens); }

int64_t scratch_floats(const AttentionArgs *a, int passes, int type, int cus, bool gradient)
{
    return by_token(a, gradient) ? 0 : attention_chunk_scratch_floats(a, passes, type, cus);
}

hipError_t launch(const AttentionArgs *a, int passes, int type, int out_type, float *scratch, int cus, bool gradient, hipStream_t st)
{
    if (!by_token(a, gradient)) return launch_attention_chunk(a, passes, type, out_type, scratch, cus, st);
    hipError_t e = hipSuccess;
    for (int i = 0; i < passes && e == hipSuccess; ++i) e = launch_attention_recurrent(a[i], type, out_type, st);
    return e;
}

// the state of `A`, kept [key][value] where its rows are keys, else read as the transpose
void from_state(AttentionArgs &A, const float *state, float *state_out, bool transposed)
{
    A.state = state;
    A.state_out = state_out;
    A.row_stride = transposed ? 1 : A.columns;
    A.column_stride = transposed ? A.rows : 1;
}

// the call for a batch that one launch holds
int forward(sig_ctx *ctx, const sig_attention_t &s, const void *q, const void *k, const void *v, const float *log_decay, const float *state,
            const int64_t *lengths, void *out, float *state_out, hipStream_t st)
{
    const int group = s.heads / s.shared_heads;
    AttentionArgs A = pass(s, log_decay, lengths, s.key_dim, s.value_dim);
    operand(&A.x, A.xs, &A.x_group, q, s.q_strides, 1);
    operand(&A.y, A.ys, &A.y_group, k, s.k_strides, group);
    operand(&A.z, A.zs, &A.z_group, v, s.v_strides, group);
    A.o = out;
    contiguous(A.os, s, s.heads, s.value_dim);
    A.out_scale = s.scale;
    from_state(A, state, state_out, false);
    Scratch scratch;
    float *work = nullptr;
    if (const int64_t floats = scratch_floats(&A, 1, s.type, ctx->num_cu, false)) {
        const int got = scratch.get(ctx, (size_t)floats * sizeof(float), st, &work);
        if (got != SIG_OK) return got;
    }
    return launch(&A, 1, s.type, s.type, work, ctx->num_cu, false, st) == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}

int backward(sig_ctx *ctx, const sig_attention_t &s, const void *q, const void *k, const void *v, const float *log_decay, const float *state,
             const int64_t *lengths, const void *grad_out, const float *grad_state, void *grad_q, void *grad_k, void *grad_v, float *grad_initial,
             hipStream_t st)
{
    const int K = s.key_dim, V = s.value_dim, group = s.heads / s.shared_heads;
    int64_t gs[3];
    contiguous(gs, s, s.heads, V);

    // the three passes: the gradients of q, k and v
    AttentionArgs a[3];
    AttentionArgs &Q = a[0], &K_ = a[1], &V_ = a[2];
    Q = pass(s, log_decay, lengths, V, K);
    operand(&Q.x, Q.xs, &Q.x_group, grad_out, gs, 1);
    operand(&Q.y, Q.ys, &Q.y_group, v, s.v_strides, group);
    operand(&Q.z, Q.zs, &Q.z_group, k, s.k_strides, group);
    Q.out_scale = s.scale;
    from_state(Q, state, nullptr, true);
    Q.o = grad_q;
    contiguous(Q.os, s, s.heads, K);
    K_ = pass(s, log_decay, lengths, V, K);
    operand(&K_.x, K_.xs, &K_.x_group, v, s.v_strides, group);
    operand(&K_.y, K_.ys, &K_.y_group, grad_out, gs, 1);
    operand(&K_.z, K_.zs, &K_.z_group, q, s.q_strides, 1);
    K_.update_scale = s.scale;
    K_.reversed = 1;
    from_state(K_, grad_state, nullptr, true);
    V_ = pass(s, log_decay, lengths, K, V);
    operand(&V_.x, V_.xs, &V_.x_group, k, s.k_strides, group);
    operand(&V_.y, V_.ys, &V_.y_group, q, s.q_strides, 1);
    operand(&V_.z, V_.zs, &V_.z_group, grad_out, gs, 1);
    V_.update_scale = s.scale;
    V_.reversed = 1;
    from_state(V_, grad_state, grad_initial, false);
    K_.o = grad_k;
    contiguous(K_.os, s, s.heads, K);
    V_.o = grad_v;
    contiguous(V_.os, s, s.heads, V);
    const int cus = ctx->num_cu;
    auto status = [](hipError_t e) { return e == hipSuccess ? SIG_OK : SIG_ERR_HIP; };
    if (s.T == 0) return status(launch(&V_, 1, s.type, s.type, nullptr, cus, true, st));      // (the state's gradient alone)

    // shared keys' and values' gradients go to scratch first, heads apart, and are added up from there
    const bool shared = group > 1;
    int64_t states = scratch_floats(a, shared ? 1 : 3, s.type, cus, true);
    if (shared) {
        const int64_t floats = scratch_floats(a + 1, 2, s.type, cus, true);
        if (floats > states) states = floats;
    }
    const int64_t parts = shared ? s.B * s.T * s.heads : 0;
    Scratch scratch;
    float *work = nullptr;
    if (states + parts > 0) {
        const int rc = scratch.get(ctx, (size_t)(states + parts * (K + V)) * sizeof(float), st, &work);
        if (rc != SIG_OK) return rc;
    }
    if (!shared) return status(launch(a, 3, s.type, s.type, work, cus, true, st));
    float *part_k = work + states, *part_v = part_k + parts * K;
    K_.o = part_k;
    V_.o = part_v;
    hipError_t e = launch(a, 1, s.type, s.type, work, cus, true, st);
    if (e == hipSuccess) e = launch(a + 1, 2, s.type, SIG_F32, work, cus, true, st);
    auto add_up = [&](const float *part, void *grad, int dim) {
        const int64_t rows = s.B * s.T * s.shared_heads;
        const int each = dim % 4 == 0 ? 4 : 1;
        int lanes = 1;
        while (lanes * each < dim) lanes *= 2;
        const int64_t blocks = (rows + kThreads / lanes - 1) / (kThreads / lanes);
        const unsigned grid = (unsigned)(blocks < 65536 ? blocks : 65536);
        with_type(s.type, [&](auto t) {
            using E = typename decltype(t)::type;
            if (each == 4) sig_attention_share_kernel<E, 4><<<grid, kThreads, 0, st>>>(part, (E *)grad, rows, group, dim, lanes);
            else sig_attention_share_kernel<E, 1><<<grid, kThreads, 0, st>>>(part, (E *)grad, rows, group, dim, lanes);
        });
        return hipGetLastError();
    };
    if (e == hipSuccess) e = add_up(part_k, grad_k, K);
    if (e == hipSuccess) e = add_up(part_v, grad_v, V);
    return status(e);
}

// p + count values of `bytes`; null stays null
template <typename P>
P *behind(P *p, int64_t count, int64_t bytes)
{
    using Byte = std::conditional_t<std::is_const_v<P>, const char, char>;
    return p ? (P *)((Byte *)p + count * bytes) : p;
}

// f(slice of the shape, its first batch element) for slices of at most `most` of them, until one fails
template <typename F>
int in_slices(const sig_attention_t &s, int64_t most, F f)
{
    sig_attention_t part = s;
    for (int64_t b = 0; b < s.B; b += most) {
        part.B = s.B - b < most ? s.B - b : most;
        if (const int rc = f(part, b)) return rc;
    }
    return SIG_OK;
}

}  // namespace

extern "C" {

int sig_linear_attention(sig_ctx *ctx, const sig_attention_t *shape, const void *q, const void *k, const void *v, const float *log_decay,
                         const float *state, const int64_t *lengths, void *out, float *state_out, void *hip_stream)
{
    const int rc = check(ctx, shape);
    if (rc != SIG_OK) return rc;
    const sig_attention_t &s = *shape;
    if (s.B == 0 || (s.T == 0 && !state_out)) return SIG_OK;
    if (!log_decay || (s.T > 0 && (!q || !k || !v || !out))) return SIG_ERR_INVALID;
    const int64_t bytes = type_bytes(s.type), state_size = (int64_t)s.heads * s.key_dim * s.value_dim;
    return in_slices(s, kMostWorkgroups / s.heads, [&](const sig_attention_t &part, int64_t b) {
        return forward(ctx, part, behind(q, b * s.q_strides[0], bytes), behind(k, b * s.k_strides[0], bytes), behind(v, b * s.v_strides[0], bytes), log_decay,
                       behind(state, b * state_size, 4), behind(lengths, b, 8), behind(out, b * s.T * s.heads * s.value_dim, bytes),
                       behind(state_out, b * state_size, 4), (hipStream_t)hip_stream);
    });
}

int sig_linear_attention_backward(sig_ctx *ctx, const sig_attention_t *shape, const void *q, const void *k, const void *v,
                                  const float *log_decay, const float *state, const int64_t *lengths, const void *grad_out,
                                  const float *grad_state, void *grad_q, void *grad_k, void *grad_v, float *grad_initial, void *hip_stream)
{
    const int rc = check(ctx, shape);
    if (rc != SIG_OK) return rc;
    const sig_attention_t &s = *shape;
    if (s.B == 0 || (s.T == 0 && !grad_initial)) return SIG_OK;
    if (!log_decay || (s.T > 0 && (!q || !k || !v || !grad_out || !grad_q || !grad_k || !grad_v))) return SIG_ERR_INVALID;
    const int64_t bytes = type_bytes(s.type), state_size = (int64_t)s.heads * s.key_dim * s.value_dim;
    int64_t most = kMostWorkgroups / s.heads;
    if (s.heads > s.shared_heads && s.T > 0) {
        const int64_t room = kMostParts / (4 * s.T * s.heads * (s.key_dim + s.value_dim));
        if (room < most) most = room < 1 ? 1 : room;
    }
    return in_slices(s, most, [&](const sig_attention_t &part, int64_t b) {
        return backward(ctx, part, behind(q, b * s.q_strides[0], bytes), behind(k, b * s.k_strides[0], bytes), behind(v, b * s.v_strides[0], bytes), log_decay,
                        behind(state, b * state_size, 4), behind(lengths, b, 8), behind(grad_out, b * s.T * s.heads * s.value_dim, bytes),
                        behind(grad_state, b * state_size, 4), behind(grad_q, b * s.T * s.heads * s.key_dim, bytes),
                        behind(grad_k, b * s.T * s.shared_heads * s.key_dim, bytes), behind(grad_v, b * s.T * s.shared_heads * s.value_dim, bytes),
                        behind(grad_initial, b * state_size, 4), (hipStream_t)hip_stream);
    });
}

}  // extern "C"
