// Linear attention on matrix instructions, C tokens at a time (sig_attention.h).
//
// With j, i the places of two tokens in a chunk of n tokens (n = C but for the last one), S the state in front of it, and e = 1 for a
// reversed pass, which decays behind a token, else 0:
//   o_i = out_scale l^(i+1-e) x_i S + out_scale update_scale sum_{j <= i} l^(i-j) (x_i . y_j) z_j
//   S  <- l^n S + update_scale sum_j l^(n-1-j+e) y_j (x) z_j
// All powers are of one head's decay and not above 1 where it decays, so nothing has to be scaled back.
//
// A workgroup holds VT columns of one head's state in registers, 16 a wavefront, as the tiles of a matrix product: they are the left
// operand of x S as they lie.  x, y and z of a chunk are staged in LDS, the next chunk's loads stay in flight in registers
// meanwhile.  The tiles of the triangle are shared out over the wavefronts and passed on through LDS, as the fragments that
// everyone reads.  Output tiles are taken as their transpose, in which a lane holds neighbouring columns of one token.
//
// A product of matrices multiplies every pair: 0 x infinity where the triangle is empty, and the parts of an infinite number.  A chunk
// whose output is not finite is therefore worked out again token by token, so that what is not a number reaches what it
// reaches in the recurrence (launches without output: the whole segment, if its state is not finite).
#ifndef SIG_ATTENTION_CHUNK_H
#define SIG_ATTENTION_CHUNK_H

#include <type_traits>

#include "sig_attention.h"
#include "sig_matrix.h"

namespace sig {

// The pieces along time that different workgroups take (A.T tokens from place `segment * segment_tokens` on)
struct ChunkArgs {
    AttentionArgs a;
    int64_t segment_tokens;     // a multiple of the chunk; at least T where there is one segment
    int segments;
    float *states;              // [segments][B][heads][rows][columns]: state-only launches write a segment's own, others read what lies before it
};

// Tiles of C tokens x W values, one after the other: global memory -> registers -> LDS (E), zeros where there is nothing.  A thread
// takes the same group of values of every ROWS-th token.  Its loads are unconditional (what is not there is read from a value
// that is, and dropped on the way to LDS), so that all are in flight at once.
template <typename T, typename E, int C, int W, int THREADS>
struct TileLoader {
    static constexpr int GROUP = 16 / (sizeof(T) > sizeof(E) ? sizeof(T) : sizeof(E));      // values of a load
    static constexpr int WIDE = W <= 64 ? 64 : W <= 128 ? 128 : 256;                        // (threads beyond W load and drop)
    static constexpr int ROWS = THREADS / (WIDE / GROUP), COUNT = C / ROWS;
    static_assert(THREADS % (WIDE / GROUP) == 0 && C % ROWS == 0);
    const T *p;          // of the next tile
    int64_t stride;      // between tokens
    int width;           // values of a token
    bool there;
    Pack<T, GROUP> held[COUNT];

    static __device__ int row() { return threadIdx.x / (WIDE / GROUP); }
    static __device__ int place() { return threadIdx.x % (WIDE / GROUP) * GROUP; }

    // token 0 of the first tile is at `tokens`
    __device__ TileLoader(const T *tokens, int64_t stride_, int width_) : stride(stride_), width(width_)
    {
        there = place() + GROUP <= width;
        p = tokens + row() * stride + (there ? place() : 0);
    }
    // the next tile, of which 1 <= n <= C tokens are there
    __device__ void load(int n)
    {
        if (width >= GROUP) {
            if (n == C) {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) held[i] = *(const Pack<T, GROUP> *)(p + i * ROWS * stride);
            } else {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) {
                    const int r = row() + i * ROWS;
                    held[i] = *(const Pack<T, GROUP> *)(p + ((r < n ? r : n - 1) - row()) * stride);
                }
            }
        }
        p += C * stride;
    }
    // the tile of the last load(n)
    __device__ void store(E *tile, int pitch, int n) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int r = row() + i * ROWS;
            const bool ok = there && r < n;
            struct alignas(GROUP * sizeof(E)) { E v[GROUP]; } values;
#pragma unroll
            for (int j = 0; j < GROUP; ++j) values.v[j] = ok ? (E)held[i].v[j] : (E)0.0f;
            if (W == WIDE || place() < W) *(decltype(values) *)(tile + r * pitch + place()) = values;
        }
        // the last values of tokens that are no whole number of groups (after the zeros of the same thread, which then reads from place 0)
        const int rest = width % GROUP, c = place();
        if (width < W && rest && c < width && c + GROUP > width) {
            const T *from = p - C * stride + c;
#pragma unroll 1
            for (int r = row(); r < n; r += ROWS, from += ROWS * stride)
#pragma unroll 1
                for (int j = 0; j < rest; ++j) tile[r * pitch + c + j] = (E)from[j];
        }
    }
};

// One token after the other, for the chunk in LDS (see above).  store(r, o_r at the lane's column)
template <bool OUTPUT, int KT, typename E, typename Store>
__device__ inline void chunk_by_token(const AttentionArgs &A, float g, int n, const E *xs, const E *ys, int kpitch, const E *zs, int vpitch,
                                      f4 (&s)[KT], int column, Store store)
{
    const int quad = threadIdx.x % 64 / 16;
    const float shrink = expm1f(g);
#pragma unroll 1
    for (int r = 0; r < n; ++r) {
        int rows = A.rows;
        asm volatile("" : "+v"(rows));      // (compared anew: the masks of all rows would not fit the scalar registers)
        const float z = A.update_scale * (float)zs[r * vpitch + column];
        float part = 0.0f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + 4 * quad + i;
                if (row >= rows) continue;
                float c = s[kt][i];
                if (!A.reversed) c = fmaf(c, shrink, c);
                c = fmaf((float)ys[r * kpitch + row], z, c);
                if (OUTPUT) part = fmaf((float)xs[r * kpitch + row], c, part);
                if (A.reversed) c = fmaf(c, shrink, c);
                s[kt][i] = c;
            }
        if (OUTPUT) {
            part += __shfl_xor(part, 16);
            part += __shfl_xor(part, 32);
            store(r, A.out_scale * part);
        }
    }
}

// T, O: types of operands and output; E: type in LDS; K: rows of the state, rounded up; VT: columns of a workgroup; PARTS: fragments that
// the state's update takes each weighted z in (Matrix<E>::EXACT: all its digits); OUTPUT: 0 for launches that only work out the
// segments' own states
template <typename T, typename O, typename E, int C, int K, int VT, int PARTS, bool OUTPUT>
__global__ __launch_bounds__(4 * VT, K <= 128 ? 2 : 1) void sig_attention_chunk_kernel(ChunkArgs G)
{
    using M = Matrix<E>;
    using Frag = typename M::Frag;
    constexpr int THREADS = 4 * VT, WAVES = VT / 16, KPITCH = K + M::PAD, VPITCH = VT + M::PAD;
    constexpr int MT = C / 16, STEPS = C / M::STEP, KSTEPS = K / M::STEP, SUB = M::SUB;
    constexpr int SPLIT = SUB == 2 ? 2 : 1;       // bfloat16 fragments of the state and of the triangle: 16 digits
    const AttentionArgs &A = G.a;
    __shared__ __attribute__((aligned(16))) E xs[OUTPUT ? C * KPITCH : 8], ys[C * KPITCH], zs[C * VPITCH];
    __shared__ Frag triangle[OUTPUT ? MT * STEPS * SPLIT * 64 : 1];
    __shared__ float after[C + 2];                // out_scale l^(i+1)
    __shared__ float gap_weight[C + 16];          // out_scale update_scale l^(i-15), zeros up to i = 14
    __shared__ float left_weight[2 * C];          // update_scale l^(C-1-i+e), zeros from i = C on

    const int64_t head = blockIdx.x % A.heads, b = blockIdx.x / A.heads;
    const int lane = threadIdx.x % 64, line = lane % 16, quad = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int c0 = blockIdx.y * VT, width = A.columns - c0, column = wave * 16 + line;     // of the workgroup, and of the lane in it
    const int64_t length = attention_length(A, b), first = (int64_t)blockIdx.z * G.segment_tokens;
    const int64_t last = first + G.segment_tokens < length && (int)blockIdx.z + 1 < G.segments ? first + G.segment_tokens : length;
    const float g = A.log_decay[head];
    const auto power = [&](int i) { return i == 0 ? 1.0f : expf((float)i * g); };
    if (OUTPUT) {
        for (int i = threadIdx.x; i < C + 2; i += THREADS) after[i] = A.out_scale * power(i);
        for (int i = threadIdx.x; i < C + 16; i += THREADS) gap_weight[i] = i < 15 ? 0.0f : A.out_scale * A.update_scale * power(i - 15);
        for (int i = threadIdx.x; i < MT * STEPS * SPLIT * 64; i += THREADS) triangle[i] = Frag{};
    }
    for (int i = threadIdx.x; i < 2 * C; i += THREADS) left_weight[i] = i < C ? A.update_scale * power(C - 1 - i + A.reversed) : 0.0f;

    // token number i of the pass is at x + i * xstep
    const int64_t start = A.reversed ? length - 1 : 0;
    const int64_t xstep = A.reversed ? -A.xs[1] : A.xs[1], ystep = A.reversed ? -A.ys[1] : A.ys[1];
    const int64_t zstep = A.reversed ? -A.zs[1] : A.zs[1], ostep = A.reversed ? -A.os[1] : A.os[1];
    const T *x = (const T *)A.x + b * A.xs[0] + head / A.x_group * A.xs[2] + start * A.xs[1];
    const T *y = (const T *)A.y + b * A.ys[0] + head / A.y_group * A.ys[2] + start * A.ys[1];
    const T *z = (const T *)A.z + b * A.zs[0] + head / A.z_group * A.zs[2] + start * A.zs[1] + c0;
    O *o = (O *)A.o + b * A.os[0] + head * A.os[2] + start * A.os[1] + c0;

    // the state: tile kt holds, in a lane, its column at rows 16 kt + 4 quad + 0..3
    f4 s[K / 16];
    const int64_t head_state = (int64_t)A.rows * A.columns, at_head = (int64_t)b * A.heads + head;
    const bool own = !OUTPUT || G.segments > 1;   // states in scratch
    const int64_t row_stride = own ? A.columns : A.row_stride, column_stride = own ? 1 : A.column_stride;
    float *at_segment = G.states + ((int64_t)blockIdx.z * A.B * A.heads + at_head) * head_state;
    if constexpr (!OUTPUT) {
#pragma unroll
        for (int kt = 0; kt < K / 16; ++kt) s[kt] = f4{};
    } else {
        const float *at = (own ? at_segment : A.state + at_head * head_state) + 4 * quad * row_stride + (c0 + column) * column_stride;
        int rows = (own || A.state) && column < width ? A.rows - 4 * quad : 0;
        asm volatile("" : "+v"(rows));
#pragma unroll
        for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[kt][i] = 16 * kt + i < rows ? at[(16 * kt + i) * row_stride] : 0.0f;
    }

    TileLoader<T, E, C, K, THREADS> xl(x + first * xstep, xstep, A.rows), yl(y + first * ystep, ystep, A.rows);
    TileLoader<T, E, C, VT, THREADS> zl(z + first * zstep, zstep, width);
    auto load = [&](int64_t t) {
        const int n = last - t < C ? (int)(last - t) : C;
        if (OUTPUT) xl.load(n);
        yl.load(n);
        zl.load(n);
    };
    if (first < last) load(first);
    __syncthreads();

    bool by_token = false;
    for (int64_t t0 = first; t0 < last; t0 += C) {
        const int n = last - t0 < C ? (int)(last - t0) : C;
        if (OUTPUT) xl.store(xs, KPITCH, n);
        yl.store(ys, KPITCH, n);
        zl.store(zs, VPITCH, n);
        __syncthreads();
        if (t0 + C < last) load(t0 + C);

        f4 out[OUTPUT ? MT : 1] = {};
        if constexpr (OUTPUT) {
            // this wavefront's tiles of the triangle: tokens 16 m + line against 16 j + 4 quad + 0..3
            for (int tile = wave; tile < MT * (MT + 1) / 2; tile += WAVES) {
                int m = 0;
#pragma unroll
                for (int i = 1; i < MT; ++i) m += tile >= i * (i + 1) / 2;
                const int j = tile - m * (m + 1) / 2;
                f4 dots = {};
#pragma unroll
                for (int kk = 0; kk < KSTEPS; ++kk)
                    dots = M::multiply(M::along_rows(ys, KPITCH, 16 * j, kk * M::STEP), M::along_rows(xs, KPITCH, 16 * m, kk * M::STEP), dots);
                float values[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = gap_weight[15 + 16 * (m - j) + line - 4 * quad - i];
                    values[i] = j < m || 4 * quad + i <= line ? w * dots[i] : 0.0f;      // (a later token may be infinite)
                }
                M::template put<SPLIT>(values, triangle + (m * STEPS + j / SUB) * SPLIT * 64 + lane, j % SUB);
            }
            // what lies before the chunk
#pragma unroll
            for (int kk = 0; kk < KSTEPS; ++kk) {
                float values[4 * SUB];
#pragma unroll
                for (int e = 0; e < 4 * SUB; ++e) values[e] = s[kk * SUB + e / 4][e % 4];
                Frag sf[SPLIT];
                M::template split<SPLIT>(values, sf);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const Frag xf = M::along_rows(xs, KPITCH, 16 * m, kk * M::STEP);
#pragma unroll
                    for (int p = 0; p < SPLIT; ++p) out[m] = M::multiply(sf[p], xf, out[m]);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) out[m] *= after[16 * m + line + 1 - A.reversed];
            __syncthreads();
        } else if (by_token) {
            chunk_by_token<false>(A, g, n, xs, ys, KPITCH, zs, VPITCH, s, column, [](int, float) {});
            __syncthreads();
            continue;
        }

        Frag zf[STEPS];
#pragma unroll
        for (int st = 0; st < STEPS; ++st) zf[st] = M::along_columns(zs, VPITCH, st * M::STEP, wave * 16);
        if constexpr (OUTPUT) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int st = 0; st * SUB <= m; ++st)
#pragma unroll
                    for (int p = 0; p < SPLIT; ++p) out[m] = M::multiply(zf[st], triangle[((m * STEPS + st) * SPLIT + p) * 64 + lane], out[m]);
            float worst = 0.0f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) worst = fmaf(out[m][i], 0.0f, worst);     // a NaN from anything that is not finite
            if (__any(!(worst == 0.0f))) {
                chunk_by_token<true>(A, g, n, xs, ys, KPITCH, zs, VPITCH, s, column, [&](int r, float value) {
                    if (quad == 0 && column < width) o[(t0 + r) * ostep + column] = from_float<O>(value);
                });
                __syncthreads();
                continue;
            }
            const int at = wave * 16 + 4 * quad;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int r = 16 * m + line;
                if (r >= n) continue;
                O *to = o + (t0 + r) * ostep + at;
                Pack<O, 4> values;
#pragma unroll
                for (int j = 0; j < 4; ++j) values.v[j] = from_float<O>(out[m][j]);
                if (at + 4 <= width) {
                    *(Pack<O, 4> *)to = values;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at + j < width) to[j] = values.v[j];
                }
            }
        }

        // the state behind the chunk.  l^n = 1 + (l^n - 1): the power itself, rounded, would drift over many chunks where little decays
        const float shrink = expm1f((float)n * g);
#pragma unroll
        for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[kt][i] = fmaf(s[kt][i], shrink, s[kt][i]);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            float values[4 * SUB];
#pragma unroll
            for (int e = 0; e < 4 * SUB; ++e)
                values[e] = M::value(zf[st], e) * left_weight[C - n + st * M::STEP + e / 4 * 16 + 4 * quad + e % 4];
            Frag wf[PARTS];
            M::template split<PARTS>(values, wf);
#pragma unroll
            for (int kt = 0; kt < K / 16; ++kt) {
                const Frag yf = M::along_columns(ys, KPITCH, st * M::STEP, 16 * kt);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) s[kt] = M::multiply(yf, wf[p], s[kt]);
            }
        }
        if constexpr (OUTPUT) {
            __syncthreads();
        } else {
            float worst = 0.0f;
            if (t0 + C >= last)
#pragma unroll
                for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) worst = fmaf(s[kt][i], 0.0f, worst);
            if (__syncthreads_or(!(worst == 0.0f))) {
                by_token = true;
#pragma unroll
                for (int kt = 0; kt < K / 16; ++kt) s[kt] = f4{};
                yl = TileLoader<T, E, C, K, THREADS>(y + first * ystep, ystep, A.rows);
                zl = TileLoader<T, E, C, VT, THREADS>(z + first * zstep, zstep, width);
                t0 = first - C;
                load(first);
            }
        }
    }

    if constexpr (OUTPUT) {
        if ((int)blockIdx.z + 1 == G.segments) {
            // behind the length
            O *rest = (O *)A.o + b * A.os[0] + head * A.os[2] + c0;
            const int left = width < VT ? width : VT;
            for (int64_t i = threadIdx.x; i < (A.T - length) * left; i += THREADS) rest[(length + i / left) * A.os[1] + i % left] = from_float<O>(0.0f);
        }
        if (own || !A.state_out) return;
    }
    float *to = (own ? at_segment : A.state_out + at_head * head_state) + 4 * quad * row_stride + (c0 + column) * column_stride;
    int rows = column < width ? A.rows - 4 * quad : 0;
    asm volatile("" : "+v"(rows));
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (16 * kt + i < rows) to[(16 * kt + i) * row_stride] = s[kt][i];
}

// The instance for `G`: vt columns a workgroup
template <typename T, typename O, typename E, int C, int PARTS, bool OUTPUT>
void launch_chunk_instance(const ChunkArgs &G, int vt, hipStream_t st)
{
    const AttentionArgs &A = G.a;
    const dim3 grid((unsigned)(A.B * A.heads), (unsigned)((A.columns + vt - 1) / vt), (unsigned)G.segments);
    auto go = [&](auto k) {
        constexpr int K = decltype(k)::value;
        constexpr int WIDE = K <= 128 ? 128 : 64;       // (registers)
        if (vt == WIDE) sig_attention_chunk_kernel<T, O, E, C, K, WIDE, PARTS, OUTPUT><<<grid, 4 * WIDE, 0, st>>>(G);
        else sig_attention_chunk_kernel<T, O, E, C, K, 64, PARTS, OUTPUT><<<grid, 256, 0, st>>>(G);
    };
    if (A.rows <= 64) go(std::integral_constant<int, 64>());
    else if (A.rows <= 128) go(std::integral_constant<int, 128>());
    else if (A.rows <= 192) go(std::integral_constant<int, 192>());
    else go(std::integral_constant<int, 256>());
}

template <typename T, typename E, int C>
void launch_chunk(const ChunkArgs &G, int vt, bool output, bool partial, hipStream_t st)
{
    constexpr int PARTS = Matrix<E>::EXACT;
    if (!output) launch_chunk_instance<T, T, E, C, PARTS, false>(G, vt, st);
    else if (partial) launch_chunk_instance<T, float, E, C, PARTS, true>(G, vt, st);
    else launch_chunk_instance<T, T, E, C, PARTS, true>(G, vt, st);
}

// one for each type of the operands, in a file of its own; partial: float32 output
void launch_chunk_f32(const ChunkArgs &G, int vt, bool output, bool partial, hipStream_t st);
void launch_chunk_bf16(const ChunkArgs &G, int vt, bool output, bool partial, hipStream_t st);
void launch_chunk_f16(const ChunkArgs &G, int vt, bool output, bool partial, hipStream_t st);

}  // namespace sig
#endif
