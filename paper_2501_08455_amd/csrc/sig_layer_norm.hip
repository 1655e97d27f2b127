// Layer norm of rows and its gradient (include/sig_sequence.h).
//
//   h = (x - mean) r,  r = 1 / sqrt(mean (x - mean)^2 + eps),  y = h weight + bias
//   grad_x = r (g - mean g - h mean(g h)) with g = grad_out weight;  grad_weight = sum grad_out h,  grad_bias = sum grad_out
//
// Bound by memory: two flops or so a byte.  Rows of up to kLongest values are read once: LANES threads hold a row in registers between its
// sums and its output, so that the variance is the mean square of what is left of the mean, without cancellation and without a
// second read.  Workgroups walk over rows, and in the gradient each thread adds up its columns' share of the
// weights' gradients on the way; a second launch adds up the workgroups' sums in their order.  Longer rows are cut into pieces that
// different workgroups take: partial sums, the rows' own numbers from them, then the output from a second read.
//
// Measured (a large copy reaches 4.9 TB/s, one that the last cache level holds 7.2): 65,536 rows of 780 bfloat16, 37 us forward (5.5 TB/s) and
// 72 + 5 us for the gradient and the weights' (4.3 TB/s); 16 rows of 1,111,110 float32, 12 + 3 + 26 us and 23 + 5 + 38 us (5.3 to 6.2 TB/s in
// the launches that read rows); 128 rows of 780, 3.6 us, which is a launch.
#include <type_traits>
#include <utility>

#include "sig_context.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;
constexpr int64_t kLongest = 16384;     // values of a row that one workgroup takes
constexpr int64_t kPiece = 8192;        // values of a piece of a longer row
constexpr int kWidest = 1024;           // workgroups that keep sums of the weights' gradients

template <typename T, int N>
__device__ inline void widen(const Pack<T, N> &pack, float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_float(pack.v[i]);
}

template <typename T, int N>
__device__ inline void load_values(const T *p, float (&v)[N])
{
    widen(load_pack<T, N>(p), v);
}

template <typename T, int N>
__device__ inline void store_values(T *p, const float (&v)[N])
{
    Pack<T, N> pack;
#pragma unroll
    for (int i = 0; i < N; ++i) pack.v[i] = from_float<T>(v[i]);
    store_pack(p, pack);
}

// weights, or `otherwise` where there are none
template <typename W, int N>
__device__ inline void load_weight(const W *p, int64_t at, float otherwise, float (&v)[N])
{
    if (p) load_values(p + at, v);
    else
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = otherwise;
}

// Which values of `width` a thread of LANES takes: R groups of N neighbours, where a group is whole, and of the last values, too few for a
// group, one.  f(Number<group>, Number<values>, offset) for each; the last ones are group R.
template <int LANES, int R, int N>
struct Share {
    int lane, groups, rest;
    int64_t width;

    __device__ explicit Share(int64_t width_) : lane(threadIdx.x % LANES), groups((int)(width_ / N)), rest((int)(width_ % N)), width(width_) {}
    template <typename F>
    __device__ void each(F f) const
    {
        whole(f, std::make_integer_sequence<int, R>());
        if (lane < rest) f(std::integral_constant<int, R>(), std::integral_constant<int, 1>(), width - rest + lane);
    }

private:
    template <typename F, int... I>
    __device__ void whole(F f, std::integer_sequence<int, I...>) const
    {
        ((I * LANES + lane < groups ? f(std::integral_constant<int, I>(), std::integral_constant<int, N>(), (int64_t)(I * LANES + lane) * N) : (void)0), ...);
    }
};

// R groups of N values and one more, as Share deals them out
template <typename V, int R, int N>
struct Held {
    V group[R][N], one[1];

    template <int I>
    __device__ auto &at()
    {
        if constexpr (I < R) return group[I];
        else return one;
    }
};
template <typename T, int R, int N>
struct HeldPacks {
    Pack<T, N> group[R];
    Pack<T, 1> one;

    template <int I>
    __device__ auto &at()
    {
        if constexpr (I < R) return group[I];
        else return one;
    }
};

// x of lane i ^ STEP, up to 8 where the lanes of a group of STEP hold the same number already (moves inside a row of 16 lanes cost no
// trip through LDS)
template <int STEP>
__device__ inline float across(float x)
{
    if constexpr (STEP > 8) return __shfl_xor(x, STEP);
    constexpr int CONTROL = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;      // quads permuted, half rows and rows mirrored
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xF, 0xF, true));
}

template <int LANES>
__device__ inline float lane_sum(float x)
{
    x += across<1>(x);
    x += across<2>(x);
    x += across<4>(x);
    if constexpr (LANES > 8) x += across<8>(x);
    if constexpr (LANES > 16) x += across<16>(x);
    if constexpr (LANES > 32) x += across<32>(x);
    return x;
}

// Sums of COUNT numbers over the LANES threads of a row, in each of them.  room: a place of its own for every second call (a workgroup
// may be one call ahead of its slowest wavefront)
template <int LANES, int COUNT>
__device__ inline void row_sums(float (&x)[COUNT], float (*room)[2][16], int turn)
{
#pragma unroll
    for (int c = 0; c < COUNT; ++c) x[c] = lane_sum<(LANES < kWave ? LANES : kWave)>(x[c]);
    if constexpr (LANES > kWave) {
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int c = 0; c < COUNT; ++c) room[turn][c][threadIdx.x / kWave] = x[c];
        __syncthreads();
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            x[c] = 0.0f;
#pragma unroll
            for (int w = 0; w < LANES / kWave; ++w) x[c] += room[turn][c][w];
        }
    }
}

template <typename T>
constexpr int kGroup = 16 / sizeof(T);     // values of a load

// LANES threads a row, R groups each
template <typename T, typename W, int LANES, int R>
__global__ __launch_bounds__(LANES > kThreads ? LANES : kThreads) void sig_layer_norm_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t width,
                                                                                             const W *weight, const W *bias, float eps, T *y, float *stats)
{
    constexpr int N = kGroup<T>, THREADS = LANES > kThreads ? LANES : kThreads, TOGETHER = THREADS / LANES;
    __shared__ float room[2][2][16];
    const Share<LANES, R, N> share(width);
    const float n = (float)width;
    const int64_t step = (int64_t)gridDim.x * TOGETHER;
    Held<float, R, N> w, b;
    HeldPacks<T, R, N> next;
    auto load = [&](int64_t row) {
        share.each([&](auto i, auto count, int64_t at) { next.template at<i()>() = load_pack<T, count()>(x + row * x_stride + at); });
    };
    share.each([&](auto i, auto, int64_t at) {
        load_weight(weight, at, 1.0f, w.template at<i()>());
        load_weight(bias, at, 0.0f, b.template at<i()>());
    });
    // the next row is loaded while this one is worked on
    int64_t row = (int64_t)blockIdx.x * TOGETHER + threadIdx.x / LANES;
    if (row < rows) load(row);
    for (; row < rows; row += step) {
        Held<float, R, N> v;
        float sum[1] = {0.0f}, squares[1] = {0.0f};
        share.each([&](auto i, auto, int64_t) { widen(next.template at<i()>(), v.template at<i()>()); });
        if (row + step < rows) load(row + step);
        share.each([&](auto i, auto, int64_t) {
            for (float value : v.template at<i()>()) sum[0] += value;
        });
        row_sums<LANES>(sum, room, 0);
        const float mean = sum[0] / n;
        share.each([&](auto i, auto, int64_t) {
            for (float &value : v.template at<i()>()) {
                value -= mean;
                squares[0] = fmaf(value, value, squares[0]);
            }
        });
        row_sums<LANES>(squares, room, 1);
        const float scale = 1.0f / sqrtf(squares[0] / n + eps);
        share.each([&](auto i, auto count, int64_t at) {
            auto &mine = v.template at<i()>();
            auto &ww = w.template at<i()>(), &bb = b.template at<i()>();
#pragma unroll
            for (int j = 0; j < count(); ++j) mine[j] = fmaf(mine[j] * scale, ww[j], bb[j]);
            store_values(y + row * width + at, mine);
        });
        if (stats && share.lane == 0) {
            stats[2 * row] = mean;
            stats[2 * row + 1] = scale;
        }
    }
}

// The gradient, LANES threads a row; sums: [gridDim.x][2][width], or null where no weight wants a gradient
template <typename T, typename W, int LANES, int R>
__global__ __launch_bounds__(LANES > kThreads ? LANES : kThreads) void sig_layer_norm_grad_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t width,
                                                                                                  const W *weight, const float *stats, const T *grad,
                                                                                                  int64_t grad_stride, T *grad_x, float *sums)
{
    constexpr int N = kGroup<T>, THREADS = LANES > kThreads ? LANES : kThreads, TOGETHER = THREADS / LANES;
    constexpr bool KEPT = LANES <= kWave;      // the weights stay in registers, and the next row is loaded while this one is worked on
    __shared__ float room[2][2][16];
    __shared__ float shares[TOGETHER > 1 ? THREADS * N : 1];
    const Share<LANES, R, N> share(width);
    const float n = (float)width;
    const int64_t step = (int64_t)gridDim.x * TOGETHER;
    Held<float, R, N> of_weight = {}, of_bias = {}, w;
    HeldPacks<T, R, N> next_x, next_g;
    float next_mean = 0.0f, next_scale = 0.0f;
    auto load = [&](int64_t row) {
        next_mean = stats[2 * row];
        next_scale = stats[2 * row + 1];
        share.each([&](auto i, auto count, int64_t at) {
            next_x.template at<i()>() = load_pack<T, count()>(x + row * x_stride + at);
            next_g.template at<i()>() = load_pack<T, count()>(grad + row * grad_stride + at);
        });
    };
    if (KEPT) share.each([&](auto i, auto, int64_t at) { load_weight(weight, at, 1.0f, w.template at<i()>()); });
    int turn = 0;
    int64_t row = (int64_t)blockIdx.x * TOGETHER + threadIdx.x / LANES;
    if (KEPT && row < rows) load(row);
    for (; row < rows; row += step) {
        const float mean = KEPT ? next_mean : stats[2 * row], scale = KEPT ? next_scale : stats[2 * row + 1];
        Held<float, R, N> h, g;
        float both[2] = {0.0f, 0.0f};
        share.each([&](auto i, auto count, int64_t at) {
            widen(KEPT ? next_x.template at<i()>() : load_pack<T, count()>(x + row * x_stride + at), h.template at<i()>());
            widen(KEPT ? next_g.template at<i()>() : load_pack<T, count()>(grad + row * grad_stride + at), g.template at<i()>());
        });
        if (KEPT && row + step < rows) load(row + step);
        share.each([&](auto i, auto count, int64_t at) {
            auto &hh = h.template at<i()>(), &gg = g.template at<i()>(), &ww = w.template at<i()>();
            auto &dw = of_weight.template at<i()>(), &db = of_bias.template at<i()>();
            if (!KEPT) load_weight(weight, at, 1.0f, ww);
#pragma unroll
            for (int j = 0; j < count(); ++j) {
                hh[j] = (hh[j] - mean) * scale;
                db[j] += gg[j];
                dw[j] = fmaf(gg[j], hh[j], dw[j]);
                gg[j] *= ww[j];
                both[0] += gg[j];
                both[1] = fmaf(gg[j], hh[j], both[1]);
            }
        });
        if (!grad_x) continue;
        row_sums<LANES>(both, room, turn);
        turn ^= 1;
        const float sum = both[0] / n, dot = both[1] / n;
        share.each([&](auto i, auto count, int64_t at) {
            auto &hh = h.template at<i()>(), &gg = g.template at<i()>();
#pragma unroll
            for (int j = 0; j < count(); ++j) gg[j] = scale * (gg[j] - sum - hh[j] * dot);
            store_values(grad_x + row * width + at, gg);
        });
    }
    if (!sums) return;
    // The workgroup's sums; where several rows share a workgroup, group by group, added up over their threads in order.  (Every thread of a
    // workgroup has the same groups to pass, if not the same values in them: the barriers are met by all.)
    float *own = sums + (int64_t)blockIdx.x * 2 * width;
    auto keep = [&](auto which) {
        auto &from = which() ? of_bias : of_weight;
        if constexpr (TOGETHER == 1) {
            share.each([&](auto i, auto, int64_t at) { store_values(own + which() * width + at, from.template at<i()>()); });
        } else {
#pragma unroll
            for (int r = 0; r <= R; ++r) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (r < R) shares[threadIdx.x * N + j] = from.group[r < R ? r : 0][j];
                    else if (j == 0) shares[threadIdx.x * N] = from.one[0];
                __syncthreads();
                const bool mine = threadIdx.x < LANES && (r < R ? r * LANES + share.lane < share.groups : share.lane < share.rest);
                if (!mine) continue;
                const int64_t at = r < R ? (int64_t)(r * LANES + share.lane) * N : width - share.rest + share.lane;
                for (int j = 0; j < (r < R ? N : 1); ++j) {
                    float sum = 0.0f;
                    for (int t = 0; t < TOGETHER; ++t) sum += shares[(t * LANES + share.lane) * N + j];
                    own[which() * width + at + j] = sum;
                }
            }
        }
    };
    keep(std::integral_constant<int, 0>());
    keep(std::integral_constant<int, 1>());
}

// grad_weight, grad_bias from [parts][2][width] sums: 1024 / LINES columns a workgroup, the parts shared out over its LINES rows of threads
template <typename W, int LINES>
__global__ __launch_bounds__(1024) void sig_layer_norm_weights_kernel(const float *sums, int64_t parts, int64_t width, W *grad_weight, W *grad_bias)
{
    constexpr int COLUMNS = 1024 / LINES;
    __shared__ float room[LINES][COLUMNS + 1];
    const int column = threadIdx.x % COLUMNS, line = threadIdx.x / COLUMNS;
    const int64_t at = (int64_t)blockIdx.x * COLUMNS + column;      // of 2 * width
    float sum = 0.0f;
    if (at < 2 * width)
#pragma unroll 4
        for (int64_t p = line; p < parts; p += LINES) sum += sums[p * 2 * width + at];
    if constexpr (LINES > 1) {
        room[line][column] = sum;
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < LINES; ++i) sum += room[i][column];
    }
    if (line || at >= 2 * width) return;
    W *to = at < width ? grad_weight : grad_bias;
    if (to) to[at < width ? at : at - width] = from_float<W>(sum);
}

// ---------------------------------------------------------------- long rows
// Numbers of a piece: its mean and the sum of squares of what is left of it
template <typename T>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_pieces_kernel(const T *x, int64_t x_stride, int64_t pieces, int64_t width, float *numbers)
{
    constexpr int N = kGroup<T>, R = kPiece / (kThreads * N);
    __shared__ float room[2][2][16];
    const int64_t row = blockIdx.x / pieces, first = blockIdx.x % pieces * kPiece, n = min(kPiece, width - first);
    const Share<kThreads, R, N> share(n);
    Held<float, R, N> v;
    float sum[1] = {0.0f}, squares[1] = {0.0f};
    share.each([&](auto i, auto, int64_t at) { load_values(x + row * x_stride + first + at, v.template at<i()>()); });
    share.each([&](auto i, auto, int64_t) {
        for (float value : v.template at<i()>()) sum[0] += value;
    });
    row_sums<kThreads>(sum, room, 0);
    const float mean = sum[0] / (float)n;
    share.each([&](auto i, auto, int64_t) {
        for (float value : v.template at<i()>()) squares[0] = fmaf(value - mean, value - mean, squares[0]);
    });
    row_sums<kThreads>(squares, room, 1);
    if (threadIdx.x == 0) {
        numbers[2 * blockIdx.x] = mean;
        numbers[2 * blockIdx.x + 1] = squares[0];
    }
}

// stats of a row from its pieces: a wavefront a row
__global__ __launch_bounds__(kThreads) void sig_layer_norm_stats_kernel(const float *numbers, int64_t rows, int64_t pieces, int64_t width, float eps, float *stats)
{
    const int64_t row = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
    if (row >= rows) return;
    const int lane = threadIdx.x % kWave;
    const float *own = numbers + 2 * row * pieces;
    // (in 64 bits: two passes over a few hundred numbers cost nothing)
    double sum = 0.0, squares = 0.0;
    for (int64_t p = lane; p < pieces; p += kWave) sum += (double)own[2 * p] * (double)min(kPiece, width - p * kPiece);
    for (int step = 1; step < kWave; step *= 2) sum += __shfl_xor(sum, step);
    const double mean = sum / (double)width;
    for (int64_t p = lane; p < pieces; p += kWave) {
        const double away = own[2 * p] - mean;
        squares += own[2 * p + 1] + away * away * (double)min(kPiece, width - p * kPiece);
    }
    for (int step = 1; step < kWave; step *= 2) squares += __shfl_xor(squares, step);
    if (lane == 0) {
        stats[2 * row] = (float)mean;
        stats[2 * row + 1] = (float)(1.0 / sqrt(squares / (double)width + (double)eps));
    }
}

template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_apply_kernel(const T *x, int64_t x_stride, int64_t pieces, int64_t width, const W *weight,
                                                                        const W *bias, const float *stats, T *y)
{
    constexpr int N = kGroup<T>, R = kPiece / (kThreads * N);
    const int64_t row = blockIdx.x / pieces, first = blockIdx.x % pieces * kPiece, n = min(kPiece, width - first);
    const float mean = stats[2 * row], scale = stats[2 * row + 1];
    Share<kThreads, R, N>(n).each([&](auto, auto count, int64_t at) {
        float v[count()], w[count()], b[count()];
        load_values(x + row * x_stride + first + at, v);
        load_weight(weight, first + at, 1.0f, w);
        load_weight(bias, first + at, 0.0f, b);
#pragma unroll
        for (int i = 0; i < count(); ++i) v[i] = fmaf((v[i] - mean) * scale, w[i], b[i]);
        store_values(y + row * width + first + at, v);
    });
}

// sums of g and g h over a piece
template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_grad_pieces_kernel(const T *x, int64_t x_stride, int64_t pieces, int64_t width, const W *weight,
                                                                              const float *stats, const T *grad, int64_t grad_stride, float *numbers)
{
    constexpr int N = kGroup<T>, R = kPiece / (kThreads * N);
    __shared__ float room[2][2][16];
    const int64_t row = blockIdx.x / pieces, first = blockIdx.x % pieces * kPiece, n = min(kPiece, width - first);
    const float mean = stats[2 * row], scale = stats[2 * row + 1];
    float both[2] = {0.0f, 0.0f};
    Share<kThreads, R, N>(n).each([&](auto, auto count, int64_t at) {
        float v[count()], g[count()], w[count()];
        load_values(x + row * x_stride + first + at, v);
        load_values(grad + row * grad_stride + first + at, g);
        load_weight(weight, first + at, 1.0f, w);
#pragma unroll
        for (int i = 0; i < count(); ++i) {
            g[i] *= w[i];
            both[0] += g[i];
            both[1] = fmaf(g[i], (v[i] - mean) * scale, both[1]);
        }
    });
    row_sums<kThreads>(both, room, 0);
    if (threadIdx.x == 0) {
        numbers[2 * blockIdx.x] = both[0];
        numbers[2 * blockIdx.x + 1] = both[1];
    }
}

// means of g and g h over a row from its pieces: a wavefront a row
__global__ __launch_bounds__(kThreads) void sig_layer_norm_grad_means_kernel(const float *numbers, int64_t rows, int64_t pieces, int64_t width, float *means)
{
    const int64_t row = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
    if (row >= rows) return;
    const int lane = threadIdx.x % kWave;
    const float *own = numbers + 2 * row * pieces;
    double sum = 0.0, dot = 0.0;
    for (int64_t p = lane; p < pieces; p += kWave) {
        sum += own[2 * p];
        dot += own[2 * p + 1];
    }
    for (int step = 1; step < kWave; step *= 2) {
        sum += __shfl_xor(sum, step);
        dot += __shfl_xor(dot, step);
    }
    if (lane == 0) {
        means[2 * row] = (float)(sum / (double)width);
        means[2 * row + 1] = (float)(dot / (double)width);
    }
}

// COUNT columns from `at` on, `together` rows of them: grad_x, and the sums of the weights' gradients, or where those are all rows (no
// sums) the gradients
template <int COUNT, typename T, typename W>
__device__ inline void grad_columns(int64_t at, const T *x, int64_t x_stride, int64_t rows, int64_t width, const W *weight, const float *stats,
                                    const float *means, const T *grad, int64_t grad_stride, T *grad_x, float *sums, int64_t together, W *grad_weight,
                                    W *grad_bias)
{
    const int64_t first = blockIdx.y * together, last = min(first + together, rows);
    float w[COUNT], of_weight[COUNT] = {}, of_bias[COUNT] = {};
    load_weight(weight, at, 1.0f, w);
#pragma unroll 4
    for (int64_t row = first; row < last; ++row) {
        const float mean = stats[2 * row], scale = stats[2 * row + 1];
        float h[COUNT], g[COUNT];
        load_values(x + row * x_stride + at, h);
        load_values(grad + row * grad_stride + at, g);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            h[i] = (h[i] - mean) * scale;
            of_bias[i] += g[i];
            of_weight[i] = fmaf(g[i], h[i], of_weight[i]);
        }
        if (!grad_x) continue;
        const float sum = means[2 * row], dot = means[2 * row + 1];
#pragma unroll
        for (int i = 0; i < COUNT; ++i) g[i] = scale * (g[i] * w[i] - sum - h[i] * dot);
        store_values(grad_x + row * width + at, g);
    }
    if (sums) {
        store_values(sums + blockIdx.y * 2 * width + at, of_weight);
        store_values(sums + blockIdx.y * 2 * width + width + at, of_bias);
    } else {
        if (grad_weight) store_values(grad_weight + at, of_weight);
        if (grad_bias) store_values(grad_bias + at, of_bias);
    }
}

// a group of columns each thread, and the last ones, too few for a group, one each
template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void sig_layer_norm_grad_columns_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t width, const W *weight,
                                                                               const float *stats, const float *means, const T *grad, int64_t grad_stride,
                                                                               T *grad_x, float *sums, int64_t together, W *grad_weight, W *grad_bias)
{
    constexpr int N = kGroup<T>;
    const int64_t place = (int64_t)blockIdx.x * kThreads + threadIdx.x, groups = width / N, rest = width % N;
    if (place < groups)
        grad_columns<N>(place * N, x, x_stride, rows, width, weight, stats, means, grad, grad_stride, grad_x, sums, together, grad_weight, grad_bias);
    else if (place < groups + rest)
        grad_columns<1>(groups * N + place - groups, x, x_stride, rows, width, weight, stats, means, grad, grad_stride, grad_x, sums, together, grad_weight,
                        grad_bias);
}

// ---------------------------------------------------------------- host
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

template <int N>
using Number = std::integral_constant<int, N>;

// f(Number<threads a row>, Number<groups each>) for rows of up to kLongest values: sixteen values a thread at most (the gradient keeps
// seven numbers for each), on one wavefront or part of it where that does (no barrier, several rows a workgroup), else on a workgroup
// (in pieces: 5,698 rows of 8,971 float32 175 us, so 95; the training pass of 3,000 rows of 16,000 308 us, so 228)
template <typename T, typename F>
void with_lanes(int64_t width, F f)
{
    constexpr int MOST = 16 / kGroup<T>;
    const int64_t groups = width / kGroup<T>;
    if (groups <= 8) f(Number<8>(), Number<1>());
    else if (groups <= 16) f(Number<16>(), Number<1>());
    else if (groups <= 32) f(Number<32>(), Number<1>());
    else if (groups <= 64) f(Number<64>(), Number<1>());
    else if (groups <= 128) f(Number<64>(), Number<2>());
    else if (MOST == 4 && groups <= 192) f(Number<64>(), Number<MOST == 4 ? 3 : 2>());
    else if (MOST == 4 && groups <= 256) f(Number<64>(), Number<MOST>());
    else if (groups <= 512) f(Number<256>(), Number<2>());
    else if (MOST == 4 && groups <= 1024) f(Number<256>(), Number<MOST>());
    else if (groups <= 512 * MOST) f(Number<512>(), Number<MOST>());
    else f(Number<1024>(), Number<MOST>());
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int launched() { return hipGetLastError() == hipSuccess ? SIG_OK : SIG_ERR_HIP; }

// A launch holds fewer than 2^32 threads: workgroups that walk over short rows are as many as the card has use for, long rows' pieces and the
// columns of the weights' gradients are one each.
bool too_large(int64_t rows, int64_t width)
{
    constexpr int64_t kMost = (int64_t)1 << 32;
    if (rows == 0) return 2 * width > kMost - 1024;
    return width > INT64_MAX / 16 / rows || (width > kLongest && ceil_div(width, kPiece) > (kMost - 1) / kThreads / rows);
}

}  // namespace

extern "C" {

int sig_layer_norm(sig_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int64_t width, int type, const void *weight,
                   const void *bias, int weight_type, double eps, void *y, float *stats, void *hip_stream)
{
    if (!valid(ctx, rows, width, type, weight_type) || !(eps >= 0.0)) return SIG_ERR_INVALID;
    if (too_large(rows, width)) return SIG_ERR_TOO_LARGE;
    if (rows == 0) return SIG_OK;
    if (!x || !y) return SIG_ERR_INVALID;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (width <= kLongest) {
        with_types(type, weight_type, [&](auto t, auto w) {
            using T = typename decltype(t)::type;
            using W = typename decltype(w)::type;
            with_lanes<T>(width, [&](auto lanes, auto loads) {
                constexpr int LANES = decltype(lanes)::value, THREADS = LANES > kThreads ? LANES : kThreads;
                const int64_t groups = ceil_div(rows, THREADS / LANES), most = (int64_t)ctx->num_cu * (16 * kThreads / THREADS);
                sig_layer_norm_kernel<T, W, LANES, decltype(loads)::value><<<(unsigned)(groups < most ? groups : most), THREADS, 0, st>>>(
                    (const T *)x, x_stride, rows, width, (const W *)weight, (const W *)bias, (float)eps, (T *)y, stats);
            });
        });
        return launched();
    }
    const int64_t pieces = ceil_div(width, kPiece);
    Scratch scratch;
    float *work = nullptr;
    const int rc = scratch.get(ctx, (size_t)(2 * rows * (pieces + 1)) * sizeof(float), st, &work);
    if (rc != SIG_OK) return rc;
    float *own = stats ? stats : work + 2 * rows * pieces;
    with_types(type, weight_type, [&](auto t, auto w) {
        using T = typename decltype(t)::type;
        using W = typename decltype(w)::type;
        sig_layer_norm_pieces_kernel<T><<<(unsigned)(rows * pieces), kThreads, 0, st>>>((const T *)x, x_stride, pieces, width, work);
        sig_layer_norm_stats_kernel<<<(unsigned)ceil_div(rows, kThreads / kWave), kThreads, 0, st>>>(work, rows, pieces, width, (float)eps, own);
        sig_layer_norm_apply_kernel<T, W><<<(unsigned)(rows * pieces), kThreads, 0, st>>>((const T *)x, x_stride, pieces, width, (const W *)weight,
                                                                                          (const W *)bias, own, (T *)y);
    });
    return launched();
}

int sig_layer_norm_backward(sig_ctx *ctx, const void *x, int64_t x_stride, int64_t rows, int64_t width, int type, const void *weight,
                            int weight_type, const float *stats, const void *grad_out, int64_t grad_stride, void *grad_x,
                            void *grad_weight, void *grad_bias, void *hip_stream)
{
    if (!valid(ctx, rows, width, type, weight_type)) return SIG_ERR_INVALID;
    if (too_large(rows, width)) return SIG_ERR_TOO_LARGE;
    if (rows > 0 && (!x || !stats || !grad_out)) return SIG_ERR_INVALID;
    const bool weights = grad_weight || grad_bias;
    if (!weights && (rows == 0 || !grad_x)) return SIG_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    const int64_t pieces = ceil_div(width, kPiece);
    const int values = type == SIG_F32 ? kGroup<float> : kGroup<bf16>;
    // workgroups that keep sums (short rows: each of several rows; long ones: rows that share a workgroup's columns)
    int64_t parts = 0, together = 1, numbers = 0;
    if (width <= kLongest) {
        int64_t groups = rows;
        with_types(type, weight_type, [&](auto t, auto) {
            with_lanes<typename decltype(t)::type>(width, [&](auto lanes, auto) {
                if (decltype(lanes)::value < kThreads) groups = ceil_div(rows, kThreads / decltype(lanes)::value);
            });
        });
        // one a unit at least, and from there on one for every eight turns, so that the sums stay a small part of the traffic
        parts = groups / 8 < kWidest ? groups / 8 : kWidest;
        if (parts < ctx->num_cu) parts = ctx->num_cu;
        if (parts > groups) parts = groups;
    } else if (rows > 0) {
        // columns alone fill the card four times over, or rows are cut too
        const int64_t across = ceil_div(width, (int64_t)kThreads * values), wanted = ceil_div(4 * (int64_t)ctx->num_cu, across);
        together = ceil_div(rows, wanted);
        if (together < 8) together = rows < 8 ? rows : 8;
        parts = ceil_div(rows, together);
        if (parts > 65535) together = ceil_div(rows, 65535), parts = ceil_div(rows, together);
        numbers = 2 * rows * (pieces + 1);
    }
    const bool direct = width > kLongest && parts == 1;      // (the columns' workgroups write the weights' gradients themselves)
    const int64_t floats = numbers + (weights && !direct ? 2 * parts * width : 0);
    Scratch scratch;
    float *work = nullptr;
    if (floats > 0) {
        const int rc = scratch.get(ctx, (size_t)floats * sizeof(float), st, &work);
        if (rc != SIG_OK) return rc;
    }
    float *sums = weights && !direct ? work + numbers : nullptr;
    with_types(type, weight_type, [&](auto t, auto w) {
        using T = typename decltype(t)::type;
        using W = typename decltype(w)::type;
        if (rows > 0 && width <= kLongest) {
            with_lanes<T>(width, [&](auto lanes, auto loads) {
                constexpr int LANES = decltype(lanes)::value, THREADS = LANES > kThreads ? LANES : kThreads;
                sig_layer_norm_grad_kernel<T, W, LANES, decltype(loads)::value><<<(unsigned)parts, THREADS, 0, st>>>(
                    (const T *)x, x_stride, rows, width, (const W *)weight, stats, (const T *)grad_out, grad_stride, (T *)grad_x, sums);
            });
        } else if (rows > 0) {
            float *means = work + 2 * rows * pieces;
            if (grad_x) {
                sig_layer_norm_grad_pieces_kernel<T, W><<<(unsigned)(rows * pieces), kThreads, 0, st>>>((const T *)x, x_stride, pieces, width, (const W *)weight,
                                                                                                        stats, (const T *)grad_out, grad_stride, work);
                sig_layer_norm_grad_means_kernel<<<(unsigned)ceil_div(rows, kThreads / kWave), kThreads, 0, st>>>(work, rows, pieces, width, means);
            }
            const dim3 grid((unsigned)ceil_div(width / kGroup<T> + width % kGroup<T>, kThreads), (unsigned)parts);
            sig_layer_norm_grad_columns_kernel<T, W><<<grid, kThreads, 0, st>>>((const T *)x, x_stride, rows, width, (const W *)weight, stats, means,
                                                                                (const T *)grad_out, grad_stride, (T *)grad_x, sums, together, (W *)grad_weight, (W *)grad_bias);
        }
        if (weights && !direct && parts > 32)
            sig_layer_norm_weights_kernel<W, 32><<<(unsigned)ceil_div(2 * width, 32), 1024, 0, st>>>(sums, parts, width, (W *)grad_weight, (W *)grad_bias);
        else if (weights && !direct)
            sig_layer_norm_weights_kernel<W, 1><<<(unsigned)ceil_div(2 * width, 1024), 1024, 0, st>>>(sums, parts, width, (W *)grad_weight, (W *)grad_bias);
    });
    return launched();
}

}  // extern "C"
