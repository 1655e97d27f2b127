// Linear attention one token after the other (sig_attention.h): the form for single tokens.
//
// Bound by memory: a token reads and writes the whole state, with two multiply-adds a value.  Each thread's part of the state is some
// rows apart in four neighbouring columns, so that loads are wide and the sum over rows needs two steps across lanes and one through
// LDS.  Measured, one token: 256 x 16 states of 128 x 128, 114 us (4.8 TB/s, a copy of that size 4.9); 128 x 4 of 64 x 64, 5.6 us.
#include "sig_attention.h"
#include "sig_types.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;
constexpr int kColumns = 64;      // of the state, a workgroup

// A workgroup holds kColumns columns of one head's state in registers: a thread N neighbouring columns of R rows, the
// rows of a thread kThreads * N / kColumns apart.  A token costs a barrier, behind which wavefront 0 adds up the rows' parts.
template <typename T, typename O, int N, int R>
__global__ __launch_bounds__(kThreads) void sig_attention_recurrent_kernel(AttentionArgs A)
{
    constexpr int LANES = kColumns / N, GROUPS = kThreads / LANES, WAVES = kThreads / kWave;
    __shared__ float parts[2][WAVES][kColumns];
    const int64_t head = blockIdx.x % A.heads, b = blockIdx.x / A.heads;
    const int c0 = blockIdx.y * kColumns, c = c0 + (int)(threadIdx.x % LANES) * N, group = threadIdx.x / LANES;
    const T *x = (const T *)A.x + b * A.xs[0] + head / A.x_group * A.xs[2];
    const T *y = (const T *)A.y + b * A.ys[0] + head / A.y_group * A.ys[2];
    const T *z = (const T *)A.z + b * A.zs[0] + head / A.z_group * A.zs[2];
    O *o = (O *)A.o + b * A.os[0] + head * A.os[2];
    const int64_t state_at = ((int64_t)b * A.heads + head) * A.rows * A.columns;
    const Decay decay(A.log_decay[head], 1.0f);
    const int64_t length = attention_length(A, b);
    const bool in = c < A.columns;    // (with N > 1 the columns are a multiple of N)

    float s[R][N];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = group + i * GROUPS;
        if (A.state && in && row < A.rows) {
            const float *from = A.state + state_at + row * A.row_stride + c * A.column_stride;
            if constexpr (N > 1) {
                const Pack<float, N> p = *(const Pack<float, N> *)from;
#pragma unroll
                for (int j = 0; j < N; ++j) s[i][j] = p.v[j];
            } else {
                s[i][0] = *from;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) s[i][j] = 0.0f;
        }
    }
    for (int64_t step = 0; step < length; ++step) {
        const int64_t t = A.reversed ? length - 1 - step : step;
        float zs[N], part[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            zs[j] = in ? A.update_scale * to_float(z[t * A.zs[1] + c + j]) : 0.0f;
            part[j] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int row = group + i * GROUPS;
            if (row >= A.rows) continue;      // (not 0 x what may be infinite)
            const float xr = to_float(x[t * A.xs[1] + row]), yr = to_float(y[t * A.ys[1] + row]);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (!A.reversed) s[i][j] = decay(s[i][j]);
                s[i][j] = fmaf(yr, zs[j], s[i][j]);
                part[j] = fmaf(xr, s[i][j], part[j]);
                if (A.reversed) s[i][j] = decay(s[i][j]);
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            for (int lane = LANES; lane < kWave; lane *= 2) part[j] += __shfl_xor(part[j], lane);
        float (*room)[kColumns] = parts[step & 1];
        if (threadIdx.x % kWave < LANES)
#pragma unroll
            for (int j = 0; j < N; ++j) room[threadIdx.x / kWave][threadIdx.x % LANES * N + j] = part[j];
        __syncthreads();
        if (threadIdx.x < kColumns && c0 + (int)threadIdx.x < A.columns) {
            float sum = 0.0f;
            for (int w = 0; w < WAVES; ++w) sum += room[w][threadIdx.x];
            o[t * A.os[1] + c0 + threadIdx.x] = from_float<O>(A.out_scale * sum);
        }
    }
    // behind the length
    const int left = min(kColumns, A.columns - c0);
    for (int64_t i = threadIdx.x; i < (A.T - length) * left; i += kThreads) o[(length + i / left) * A.os[1] + c0 + i % left] = from_float<O>(0.0f);
    if (!A.state_out || !in) return;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = group + i * GROUPS;
        if (row >= A.rows) continue;
        float *to = A.state_out + state_at + row * A.row_stride + c * A.column_stride;
        if constexpr (N > 1) {
            Pack<float, N> p;
#pragma unroll
            for (int j = 0; j < N; ++j) p.v[j] = s[i][j];
            *(Pack<float, N> *)to = p;
        } else {
            *to = s[i][0];
        }
    }
}

template <typename T, typename O, int N>
void launch(const AttentionArgs &A, hipStream_t st)
{
    constexpr int GROUPS = kThreads * N / kColumns;
    const dim3 grid((unsigned)(A.B * A.heads), (unsigned)((A.columns + kColumns - 1) / kColumns));
    const int rows = (A.rows + GROUPS - 1) / GROUPS;
    if (rows <= 256 / GROUPS / 16) sig_attention_recurrent_kernel<T, O, N, 256 / GROUPS / 16><<<grid, kThreads, 0, st>>>(A);
    else if (rows <= 256 / GROUPS / 4) sig_attention_recurrent_kernel<T, O, N, 256 / GROUPS / 4><<<grid, kThreads, 0, st>>>(A);
    else if (rows <= 256 / GROUPS / 2) sig_attention_recurrent_kernel<T, O, N, 256 / GROUPS / 2><<<grid, kThreads, 0, st>>>(A);
    else sig_attention_recurrent_kernel<T, O, N, 256 / GROUPS><<<grid, kThreads, 0, st>>>(A);
}

}  // namespace

namespace sig {

hipError_t launch_attention_recurrent(const AttentionArgs &A, int type, int out_type, hipStream_t st)
{
    const bool packed = A.columns % 4 == 0 && (A.column_stride == 1 || (!A.state && !A.state_out));
    with_type(type, [&](auto tag) {
        using T = typename decltype(tag)::type;
        if (out_type == type) packed ? launch<T, T, 4>(A, st) : launch<T, T, 1>(A, st);
        else packed ? launch<T, float, 4>(A, st) : launch<T, float, 1>(A, st);
    });
    return hipGetLastError();
}

}  // namespace sig
