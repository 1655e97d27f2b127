// Rotary positions (include/sig_sequence.h).
//
// Bound by memory: each value is read and written once.  A workgroup takes a few tokens.  It works out their cosines and sines once
// for all heads, in LDS, and then walks over the heads, several lines of N-value loads in flight a thread.  Measured: 4 x 8,192 tokens, 24 heads
// of 128 bfloat16, 64 turned, 88 us (4.5 TB/s, a copy of that size 4.9); 128 tokens, 16 heads of 64, 4 us, which is a launch.
#include <type_traits>

#include "sig_context.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 16;      // of a workgroup
constexpr int kTable = 2048;         // pairs of a workgroup's tokens

template <typename T>
constexpr int kGroup = 16 / sizeof(T);     // values of the widest load

struct RotaryArgs {
    int64_t B, T, heads, dim, turned;
    int64_t xs[3], ys[3], ps[2];     // strides: batch, token, head
    const void *positions;
    int position_type;
    const double *frequencies;
    float scale;
    int inverse, copy;               // copy: whether the components behind the turned ones are written
    int tokens;                      // of a workgroup
    int places;                      // threads of a line, a power of two
};

__device__ double position_of(const RotaryArgs &A, int64_t b, int64_t t)
{
    const int64_t at = b * A.ps[0] + t * A.ps[1];
    switch (A.position_type) {
    case SIG_POSITION_I32: return (double)((const int32_t *)A.positions)[at];
    case SIG_POSITION_I64: return (double)((const int64_t *)A.positions)[at];
    case SIG_POSITION_F32: return (double)((const float *)A.positions)[at];
    default: return ((const double *)A.positions)[at];
    }
}

// cos and sin of position * frequency.  The turns are reduced in 64 bits: a position of a million times a frequency of one
// radian has no digit left behind the point in 32.
__device__ void turn(double position, double frequency, float *c, float *s)
{
    const double turns = position * (frequency * 0.15915494309189535);
    sincospif(2.0f * (float)(turns - rint(turns)), s, c);
}

// N neighbouring values, or N pairs of the half layout, are a turned unit, M neighbouring values a copied one; a line is a token's head, its
// turned units first.  The last copied unit ends with the line, if that means that it overlaps the one before, or, where there are fewer
// than M values to copy, is those.  `places` threads take a line.  (Copied values in the turned units' width: 10 and 20 of 40 and 20 of 80 bfloat16
// turned 416, 118 and 202 us, so 125, 92 and 100.)
template <typename T, int N, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void sig_rotary_kernel(const T *x, T *y, RotaryArgs A)
{
    constexpr int AT_ONCE = 4;       // lines a thread has in flight
    constexpr int M = kGroup<T>;
    __shared__ float2 table[kTable];
    __shared__ int64_t from[kMostTokens], to[kMostTokens];
    const int half = (int)A.turned / 2, dim = (int)A.dim, turned = (int)A.turned, heads = (int)A.heads;
    const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * A.tokens, all = A.B * A.T;
    if (first >= all) return;
    const int tokens = all - first < A.tokens ? (int)(all - first) : A.tokens;
    for (int i = threadIdx.x; i < tokens * half || i < tokens; i += kThreads) {
        if (i < tokens) {
            const int64_t b = (first + i) / A.T, t = (first + i) % A.T;
            from[i] = b * A.xs[0] + t * A.xs[1];
            to[i] = b * A.ys[0] + t * A.ys[1];
        }
        if (i < tokens * half) {
            const int64_t token = first + i / half;
            float c, s;
            turn(position_of(A, token / A.T, token % A.T), A.frequencies[i % half], &c, &s);
            table[i] = make_float2(A.scale * c, A.inverse ? -A.scale * s : A.scale * s);
        }
    }
    __syncthreads();
    const int turned_units = INTERLEAVED ? turned / N : half / N, units = turned_units + (A.copy ? (dim - turned + M - 1) / M : 0);
    const int line_step = kThreads / A.places, token_step = line_step / heads, head_step = line_step % heads;
    const int first_line = threadIdx.x / A.places;
    for (int unit = threadIdx.x % A.places; unit < units; unit += A.places) {
        const bool copied = unit >= turned_units;
        const bool few = copied && dim - turned < M;
        const int at = !copied ? unit * N : few ? turned : min(turned + (unit - turned_units) * M, dim - M);
        int token = first_line / heads, head = first_line % heads;
        while (token < tokens) {
            Pack<T, N> low[AT_ONCE], high[AT_ONCE];
            Pack<T, M> same[N < M ? AT_ONCE : 1];      // (else `low`)
            const T *source[AT_ONCE];
            int tokens_of[AT_ONCE], heads_of[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                tokens_of[k] = token;
                heads_of[k] = head;
                token += token_step;
                head += head_step;
                if (head >= heads) {
                    head -= heads;
                    ++token;
                }
                if (tokens_of[k] >= tokens) continue;
                source[k] = x + from[tokens_of[k]] + heads_of[k] * A.xs[2] + at;
                if (N < M && copied) {
                    if (!few) same[N < M ? k : 0] = load_pack<T, M>(source[k]);
                } else if (!few) {
                    low[k] = load_pack<T, N>(source[k]);
                    if (!INTERLEAVED && !copied) high[k] = load_pack<T, N>(source[k] + half);
                }
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                if (tokens_of[k] >= tokens) continue;
                T *p = y + to[tokens_of[k]] + heads_of[k] * A.ys[2] + at;
                if (few) {
                    for (int j = 0; j < dim - turned; ++j) p[j] = source[k][j];
                } else if (copied) {
                    if constexpr (N < M) store_pack(p, same[k]);
                    else store_pack(p, low[k]);
                } else if constexpr (INTERLEAVED) {
                    const float2 *angle = table + tokens_of[k] * half + at / 2;
#pragma unroll
                    for (int j = 0; j < N; j += 2) {
                        const float a = to_float(low[k].v[j]), b = to_float(low[k].v[j + 1]), c = angle[j / 2].x, s = angle[j / 2].y;
                        low[k].v[j] = from_float<T>(a * c - b * s);
                        low[k].v[j + 1] = from_float<T>(a * s + b * c);
                    }
                    store_pack(p, low[k]);
                } else {
                    const float2 *angle = table + tokens_of[k] * half + at;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float a = to_float(low[k].v[j]), b = to_float(high[k].v[j]), c = angle[j].x, s = angle[j].y;
                        low[k].v[j] = from_float<T>(a * c - b * s);
                        high[k].v[j] = from_float<T>(a * s + b * c);
                    }
                    store_pack(p, low[k]);
                    store_pack(p + half, high[k]);
                }
            }
        }
    }
}

}  // namespace

extern "C" int sig_rotary(sig_ctx *ctx, const void *x, const int64_t *x_strides, void *y, const int64_t *y_strides, int type, int64_t B, int64_t T,
                          int64_t heads, int64_t dim, int64_t turned, const void *positions, int position_type, const int64_t *position_strides,
                          const double *frequencies, int interleaved, double scale, int inverse, void *hip_stream)
{
    if (!ctx || B < 0 || T < 0 || heads < 0 || dim < 1 || turned < 0 || turned > dim || turned % 2 || !valid_type(type) ||
        position_type < SIG_POSITION_I32 || position_type > SIG_POSITION_F64)
        return SIG_ERR_INVALID;
    if (B == 0 || T == 0 || heads == 0) return SIG_OK;
    if (!x || !y || !positions || !position_strides || (turned && !frequencies)) return SIG_ERR_INVALID;
    if (dim > INT32_MAX || heads > INT32_MAX / kMostTokens || dim * heads > INT32_MAX || B > INT32_MAX / T) return SIG_ERR_TOO_LARGE;
    if (turned / 2 > kTable) return SIG_ERR_UNSUPPORTED;
    RotaryArgs A = {B, T, heads, dim, turned, {T * heads * dim, heads * dim, dim}, {T * heads * dim, heads * dim, dim},
                    {position_strides[0], position_strides[1]}, positions, position_type, frequencies, (float)scale, inverse != 0, 1, 1, 1};
    for (int i = 0; i < 3; ++i) {
        if (x_strides) A.xs[i] = x_strides[i];
        if (y_strides) A.ys[i] = y_strides[i];
    }
    A.copy = x != y;
    // tokens that share a workgroup: as many as leave eight workgroups a unit
    const int64_t share = B * T / (8 * (int64_t)ctx->num_cu), room = turned ? kTable / (turned / 2) : kMostTokens;
    A.tokens = (int)(share < 1 ? 1 : share < kMostTokens ? share : kMostTokens);
    if (A.tokens > room) A.tokens = (int)room;
    // (a launch holds fewer than 2^32 threads along an axis)
    const int64_t blocks = (B * T + A.tokens - 1) / A.tokens, most = ((int64_t)1 << 31) / kThreads;
    const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)((blocks + most - 1) / most));
    with_type(type, [&](auto t) {
        using E = typename decltype(t)::type;
        auto go = [&](auto n) {
            constexpr int N = decltype(n)::value, M = kGroup<E>;
            const int64_t units = (interleaved ? turned / N : turned / 2 / N) + (A.copy ? (dim - turned + M - 1) / M : 0);
            while (A.places < units && A.places < kThreads) A.places *= 2;
            if (interleaved) sig_rotary_kernel<E, N, true><<<grid, kThreads, 0, (hipStream_t)hip_stream>>>((const E *)x, (E *)y, A);
            else sig_rotary_kernel<E, N, false><<<grid, kThreads, 0, (hipStream_t)hip_stream>>>((const E *)x, (E *)y, A);
        };
        // the widest loads that the turned components are a whole number of
        constexpr int MOST = kGroup<E>;
        const int64_t whole = interleaved ? turned : turned / 2;
        if (whole % MOST == 0) go(std::integral_constant<int, MOST>());
        else if (whole % (MOST / 2) == 0) go(std::integral_constant<int, MOST / 2>());
        else if (whole % 2 == 0) go(std::integral_constant<int, 2>());
        else go(std::integral_constant<int, 1>());
    });
    return hipGetLastError() == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}
