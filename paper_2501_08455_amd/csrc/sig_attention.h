// Linear attention with a decay for each head: what its entry points and kernels share.
//
// Every pass is one form.  For each batch element and head, with l = exp(log_decay) and n tokens in order
// (or, `reversed`, from the last one to the first):
//   C_i = l C_{i-1} + update_scale y_i (x) z_i,   o_i = out_scale x_i C_i
// forward:       x, y, z = q, k, v, from the initial state;
// gradient of q: x, y, z = grad_out, v, k, from the initial state's transpose;
// gradient of k: reversed, v, grad_out, q, from the transpose of the final state's gradient;
// gradient of v: reversed, k, q, grad_out, from the final state's gradient, and what is left is the initial state's.
// A reversed pass decays behind a token instead of in front of it (C_i = C + y (x) z; o_i; C = l C_i).
#ifndef SIG_ATTENTION_H
#define SIG_ATTENTION_H

#include <cfloat>

#include "sig_internal.h"
#include "sig_sequence.h"

namespace sig {

struct AttentionArgs {
    const void *x, *y, *z;             // [B][T][heads / group][rows or columns], last axis contiguous
    int64_t xs[3], ys[3], zs[3], os[3];   // strides in values: batch, token, head
    int x_group, y_group, z_group;     // heads that read one head of the operand
    void *o;
    const float *log_decay;            // [heads]
    const float *state;                // [B][heads][rows * columns], or null: zeros
    float *state_out;                  // or null; may be `state`
    int64_t row_stride, column_stride;    // of both, in floats
    const int64_t *lengths;            // [B], or null: T
    int64_t B, T;
    int heads, rows, columns;          // of the state: x and y have `rows` values, z and o `columns`
    float out_scale, update_scale;
    int reversed;
};

__device__ inline int64_t attention_length(const AttentionArgs &A, int64_t b)
{
    if (!A.lengths) return A.T;
    const int64_t n = A.lengths[b];
    return n < 0 ? 0 : n > A.T ? A.T : n;
}

// What a number is multiplied with over `tokens` tokens: l^tokens = 1 + shrink.  (The power itself, rounded, would drift over many tokens where
// little decays.)  s l^tokens is s + s shrink, where an infinite s has to stay what it is, as long as l is not 0: the s that is shrunk is
// taken into -most .. most.
struct Decay {
    float shrink, most;

    __device__ Decay(float log_decay, float tokens) : shrink(expm1f(tokens * log_decay)), most(log_decay == -INFINITY ? INFINITY : FLT_MAX) {}
    __device__ float operator()(float s) const { return fmaf(__builtin_amdgcn_fmed3f(s, -most, most), shrink, s); }
};

// types of the operands and of `o` (enum sig_type)
// one token after the other
hipError_t launch_attention_recurrent(const AttentionArgs &A, int type, int out_type, hipStream_t st);

// Passes over the same tokens in chunks (sig_attention_chunk.h), together where they hold states of the same size: floats of scratch that
// the launches need, and the launches
int64_t attention_chunk_scratch_floats(const AttentionArgs *a, int passes, int type, int cus);
hipError_t launch_attention_chunk(const AttentionArgs *a, int passes, int type, int out_type, float *scratch, int cus, hipStream_t st);

}  // namespace sig
#endif
