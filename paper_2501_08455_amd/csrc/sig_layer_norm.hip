// Layer norm of rows and its gradient (include/sig_sequence.h).
#include "sig_context.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;

// sum of `x` over the workgroup, in every thread; `room` holds a float for each wavefront
__device__ float block_sum(float x, float *room)
{
    for (int step = 32; step > 0; step >>= 1) x += __shfl_xor(x, step);
    __syncthreads();
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = x;
    __syncthreads();
    x = 0.0f;
    for (int w = 0; w < (int)blockDim.x / kWave; ++w) x += room[w];
    return x;
}

// A row in a workgroup.  The variance is the mean square of what is left of the mean: no cancellation.
template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t width, const W *weight,
                                                                  const W *bias, float eps, T *y, float *stats)
{
    __shared__ float room[kThreads / kWave];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *xr = x + row * x_stride;
        float sum = 0.0f, squares = 0.0f;
        for (int64_t i = threadIdx.x; i < width; i += kThreads) sum += to_float(xr[i]);
        const float mean = block_sum(sum, room) / (float)width;
        for (int64_t i = threadIdx.x; i < width; i += kThreads) {
            const float c = to_float(xr[i]) - mean;
            squares += c * c;
        }
        const float r = 1.0f / sqrtf(block_sum(squares, room) / (float)width + eps);
        for (int64_t i = threadIdx.x; i < width; i += kThreads) {
            const float h = (to_float(xr[i]) - mean) * r;
            y[row * width + i] = from_float<T>(h * (weight ? to_float(weight[i]) : 1.0f) + (bias ? to_float(bias[i]) : 0.0f));
        }
        if (stats && threadIdx.x == 0) {
            stats[2 * row] = mean;
            stats[2 * row + 1] = r;
        }
    }
}

template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_grad_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t width, const W *weight,
                                                                       const float *stats, const T *grad, int64_t grad_stride, T *grad_x)
{
    __shared__ float room[kThreads / kWave];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *xr = x + row * x_stride, *gr = grad + row * grad_stride;
        const float mean = stats[2 * row], r = stats[2 * row + 1];
        float sum = 0.0f, dot = 0.0f;
        for (int64_t i = threadIdx.x; i < width; i += kThreads) {
            const float g = to_float(gr[i]) * (weight ? to_float(weight[i]) : 1.0f);
            sum += g;
            dot += g * ((to_float(xr[i]) - mean) * r);
        }
        sum = block_sum(sum, room) / (float)width;
        dot = block_sum(dot, room) / (float)width;
        for (int64_t i = threadIdx.x; i < width; i += kThreads) {
            const float g = to_float(gr[i]) * (weight ? to_float(weight[i]) : 1.0f);
            grad_x[row * width + i] = from_float<T>(r * (g - sum - dot * ((to_float(xr[i]) - mean) * r)));
        }
    }
}

// Gradients of the weights: 64 columns a workgroup, rows taken in turn by its wavefronts
template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_weights_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t width,
                                                                          const float *stats, const T *grad, int64_t grad_stride,
                                                                          W *grad_weight, W *grad_bias)
{
    __shared__ float room[2][kThreads];
    const int64_t i = (int64_t)blockIdx.x * kWave + threadIdx.x % kWave;
    float dw = 0.0f, db = 0.0f;
    if (i < width)
        for (int64_t row = threadIdx.x / kWave; row < rows; row += kThreads / kWave) {
            const float g = to_float(grad[row * grad_stride + i]);
            dw += g * ((to_float(x[row * x_stride + i]) - stats[2 * row]) * stats[2 * row + 1]);
            db += g;
        }
    room[0][threadIdx.x] = dw;
    room[1][threadIdx.x] = db;
    __syncthreads();
    if (threadIdx.x >= kWave || i >= width) return;
    for (int w = 1; w < kThreads / kWave; ++w) {
        dw += room[0][threadIdx.x + w * kWave];
        db += room[1][threadIdx.x + w * kWave];
    }
    if (grad_weight) grad_weight[i] = from_float<W>(dw);
    if (grad_bias) grad_bias[i] = from_float<W>(db);
}

bool valid(const sig_ctx *ctx, int64_t rows, int64_t width, int type, int weight_type)
{
    return ctx && rows >= 0 && width >= 1 && valid_type(type) && (weight_type == SIG_F32 || weight_type == type);
}

// f(Tag<value type>, Tag<weight type>)
template <typename F>
void with_types(int type, int weight_type, F f)
{
    with_type(type, [&](auto tag) {
        if (weight_type == type) f(tag, tag);
        else f(tag, Tag<float>());
    });
}

int launched() { return hipGetLastError() == hipSuccess ? SIG_OK : SIG_ERR_HIP; }

}  // namespace

extern "C" {

int sig_layer_norm(sig_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int64_t width, int type, const void *weight,
                   const void *bias, int weight_type, double eps, void *y, float *stats, void *hip_stream)
{
    if (!valid(ctx, rows, width, type, weight_type) || !(eps >= 0.0)) return SIG_ERR_INVALID;
    if (rows > 0 && width > INT64_MAX / 8 / rows) return SIG_ERR_TOO_LARGE;
    if (rows == 0) return SIG_OK;
    if (!x || !y) return SIG_ERR_INVALID;
    const unsigned grid = (unsigned)(rows < (1 << 20) ? rows : 1 << 20);
    with_types(type, weight_type, [&](auto t, auto w) {
        using T = typename decltype(t)::type;
        using W = typename decltype(w)::type;
        sig_layer_norm_kernel<T, W><<<grid, kThreads, 0, (hipStream_t)hip_stream>>>((const T *)x, x_stride, rows, width, (const W *)weight, (const W *)bias,
                                                                                    (float)eps, (T *)y, stats);
    });
    return launched();
}

int sig_layer_norm_backward(sig_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int64_t width, int type, const void *weight,
                            int weight_type, const float *stats, const void *grad_out, int64_t grad_stride, void *grad_x,
                            void *grad_weight, void *grad_bias, void *hip_stream)
{
    if (!valid(ctx, rows, width, type, weight_type)) return SIG_ERR_INVALID;
    if (rows > 0 && width > INT64_MAX / 8 / rows) return SIG_ERR_TOO_LARGE;
    if (rows > 0 && (!x || !stats || !grad_out)) return SIG_ERR_INVALID;
    const hipStream_t st = (hipStream_t)hip_stream;
    const unsigned grid = (unsigned)(rows < (1 << 20) ? rows : 1 << 20);
    if ((width + kWave - 1) / kWave > INT32_MAX) return SIG_ERR_TOO_LARGE;
    with_types(type, weight_type, [&](auto t, auto w) {
        using T = typename decltype(t)::type;
        using W = typename decltype(w)::type;
        if (grad_x && rows > 0)
            sig_layer_norm_grad_kernel<T, W><<<grid, kThreads, 0, st>>>((const T *)x, x_stride, rows, width, (const W *)weight, stats,
                                                                        (const T *)grad_out, grad_stride, (T *)grad_x);
        if (grad_weight || grad_bias)
            sig_layer_norm_weights_kernel<T, W><<<(unsigned)((width + kWave - 1) / kWave), kThreads, 0, st>>>(
                (const T *)x, x_stride, rows, width, stats, (const T *)grad_out, grad_stride, (W *)grad_weight, (W *)grad_bias);
    });
    return launched();
}

}  // extern "C"
