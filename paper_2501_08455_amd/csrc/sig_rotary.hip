// Rotary positions (include/sig_sequence.h).
#include "sig_context.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
    int64_t B, T, heads, dim, turned;
    int64_t xs[3], ys[3], ps[2];     // strides: batch, token, head
    const void *positions;
    int position_type;
    const double *frequencies;
    float scale;
    int interleaved, inverse;
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

// A thread takes a pair, or one of the components that are copied.
template <typename T>
__global__ __launch_bounds__(kThreads) void sig_rotary_kernel(const T *x, T *y, RotaryArgs A)
{
    const int64_t half = A.turned / 2, slots = half + (A.dim - A.turned);
    const int64_t token = blockIdx.x, b = token / A.T, t = token % A.T;
    const double position = position_of(A, b, t);
    for (int64_t j = threadIdx.x; j < slots * A.heads; j += kThreads) {
        const int64_t h = j / slots, i = j % slots;
        const T *xr = x + b * A.xs[0] + t * A.xs[1] + h * A.xs[2];
        T *yr = y + b * A.ys[0] + t * A.ys[1] + h * A.ys[2];
        if (i >= half) {
            yr[i + half] = xr[i + half];
            continue;
        }
        const int64_t first = A.interleaved ? 2 * i : i, second = A.interleaved ? 2 * i + 1 : i + half;
        float c, s;
        turn(position, A.frequencies[i], &c, &s);
        if (A.inverse) s = -s;
        const float p = to_float(xr[first]), q = to_float(xr[second]);
        yr[first] = from_float<T>(A.scale * (p * c - q * s));
        yr[second] = from_float<T>(A.scale * (p * s + q * c));
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
    if (dim > INT32_MAX || heads > INT32_MAX || dim * heads > INT32_MAX || B > INT32_MAX / T) return SIG_ERR_TOO_LARGE;
    RotaryArgs A = {B, T, heads, dim, turned, {T * heads * dim, heads * dim, dim}, {T * heads * dim, heads * dim, dim},
                    {position_strides[0], position_strides[1]}, positions, position_type, frequencies, (float)scale, interleaved != 0, inverse != 0};
    for (int i = 0; i < 3; ++i) {
        if (x_strides) A.xs[i] = x_strides[i];
        if (y_strides) A.ys[i] = y_strides[i];
    }
    with_type(type, [&](auto t) {
        using E = typename decltype(t)::type;
        sig_rotary_kernel<E><<<(unsigned)(B * T), kThreads, 0, (hipStream_t)hip_stream>>>((const E *)x, (E *)y, A);
    });
    return hipGetLastError() == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}
