// Entry points of linear attention (include/sig_sequence.h): argument checks, the passes of the gradient, and the sum
// over heads that share keys and values.
#include "sig_attention.h"
#include "sig_context.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;
constexpr int kMostDim = 256;

// out[token][shared head][.] = sum over the heads of a shared head of part[token][head][.], in their order
template <typename T>
__global__ __launch_bounds__(kThreads) void sig_attention_share_kernel(const float *part, T *out, int64_t values, int group, int dim)
{
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < values; i += (int64_t)gridDim.x * kThreads) {
        const float *p = part + i / dim * group * dim + i % dim;
        float sum = 0.0f;
        for (int h = 0; h < group; ++h) sum += p[(int64_t)h * dim];
        out[i] = from_float<T>(sum);
    }
}

int check(const sig_ctx *ctx, const sig_attention_t *s)
{
    if (!ctx || !s || s->B < 0 || s->T < 0 || s->heads < 1 || s->shared_heads < 1 || s->heads % s->shared_heads || s->key_dim < 1 ||
        s->value_dim < 1 || !valid_type(s->type))
        return SIG_ERR_INVALID;
    if (s->key_dim > kMostDim || s->value_dim > kMostDim) return SIG_ERR_UNSUPPORTED;
    if (s->B > INT32_MAX / s->heads || (s->T > 0 && s->B * s->heads > INT64_MAX / (8 * kMostDim) / s->T)) return SIG_ERR_TOO_LARGE;
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

// the state of `A`, kept [key][value] where its rows are keys, else read as the transpose
void from_state(AttentionArgs &A, const float *state, float *state_out, bool transposed)
{
    A.state = state;
    A.state_out = state_out;
    A.row_stride = transposed ? 1 : A.columns;
    A.column_stride = transposed ? A.rows : 1;
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
    const int group = s.heads / s.shared_heads;
    AttentionArgs A = pass(s, log_decay, lengths, s.key_dim, s.value_dim);
    operand(&A.x, A.xs, &A.x_group, q, s.q_strides, 1);
    operand(&A.y, A.ys, &A.y_group, k, s.k_strides, group);
    operand(&A.z, A.zs, &A.z_group, v, s.v_strides, group);
    A.o = out;
    contiguous(A.os, s, s.heads, s.value_dim);
    A.out_scale = s.scale;
    from_state(A, state, state_out, false);
    return launch_attention_recurrent(A, s.type, s.type, (hipStream_t)hip_stream) == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}

int sig_linear_attention_backward(sig_ctx *ctx, const sig_attention_t *shape, const void *q, const void *k, const void *v,
                                  const float *log_decay, const float *state, const int64_t *lengths, const void *grad_out,
                                  const float *grad_state, void *grad_q, void *grad_k, void *grad_v, float *grad_initial, void *hip_stream)
{
    int rc = check(ctx, shape);
    if (rc != SIG_OK) return rc;
    const sig_attention_t &s = *shape;
    if (s.B == 0 || (s.T == 0 && !grad_initial)) return SIG_OK;
    if (!log_decay || (s.T > 0 && (!q || !k || !v || !grad_out || !grad_q || !grad_k || !grad_v))) return SIG_ERR_INVALID;
    const hipStream_t st = (hipStream_t)hip_stream;
    const int K = s.key_dim, V = s.value_dim, group = s.heads / s.shared_heads;
    int64_t gs[3];
    contiguous(gs, s, s.heads, V);

    Scratch scratch;
    float *part = nullptr;
    if (group > 1 && s.T > 0) {
        rc = scratch.get(ctx, (size_t)(s.B * s.T * s.heads) * (K > V ? K : V) * sizeof(float), st, &part);
        if (rc != SIG_OK) return rc;
    }
    // the gradient of shared keys or values: heads apart in scratch, then their sum
    auto shared_pass = [&](AttentionArgs &A, void *grad, int dim) {
        A.o = part ? (void *)part : grad;
        contiguous(A.os, s, s.heads, dim);
        hipError_t e = launch_attention_recurrent(A, s.type, part ? (int)SIG_F32 : s.type, st);
        if (e != hipSuccess || !part) return e;
        const int64_t values = s.B * s.T * s.shared_heads * dim, blocks = (values + kThreads - 1) / kThreads;
        with_type(s.type, [&](auto t) {
            using E = typename decltype(t)::type;
            sig_attention_share_kernel<E><<<(unsigned)(blocks < 65536 ? blocks : 65536), kThreads, 0, st>>>(part, (E *)grad, values, group, dim);
        });
        return hipGetLastError();
    };

    hipError_t e = hipSuccess;
    if (s.T > 0) {
        AttentionArgs A = pass(s, log_decay, lengths, V, K);
        operand(&A.x, A.xs, &A.x_group, grad_out, gs, 1);
        operand(&A.y, A.ys, &A.y_group, v, s.v_strides, group);
        operand(&A.z, A.zs, &A.z_group, k, s.k_strides, group);
        A.out_scale = s.scale;
        from_state(A, state, nullptr, true);
        A.o = grad_q;
        contiguous(A.os, s, s.heads, K);
        e = launch_attention_recurrent(A, s.type, s.type, st);
    }
    if (e == hipSuccess && s.T > 0) {
        AttentionArgs A = pass(s, log_decay, lengths, V, K);
        operand(&A.x, A.xs, &A.x_group, v, s.v_strides, group);
        operand(&A.y, A.ys, &A.y_group, grad_out, gs, 1);
        operand(&A.z, A.zs, &A.z_group, q, s.q_strides, 1);
        A.update_scale = s.scale;
        A.reversed = 1;
        from_state(A, grad_state, nullptr, true);
        e = shared_pass(A, grad_k, K);
    }
    if (e == hipSuccess) {
        AttentionArgs A = pass(s, log_decay, lengths, K, V);
        operand(&A.x, A.xs, &A.x_group, k, s.k_strides, group);
        operand(&A.y, A.ys, &A.y_group, q, s.q_strides, 1);
        operand(&A.z, A.zs, &A.z_group, grad_out, gs, 1);
        A.update_scale = s.scale;
        A.reversed = 1;
        from_state(A, grad_state, grad_initial, false);
        e = shared_pass(A, grad_v, V);
    }
    return e == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}

}  // extern "C"
