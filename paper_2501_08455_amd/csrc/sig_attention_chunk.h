// Linear attention on matrix instructions, C tokens at a time (sig_attention.h).
//
// With j, i the places of two tokens in a chunk of n tokens (n = C but for the last one), S the state in front of it, and e = 1 for a
// reversed pass, which decays behind a token, else 0:
//   o_i = out_scale l^(i+1-e) x_i S + out_scale update_scale sum_{j <= i} l^(i-j) (x_i . y_j) z_j
//   S  <- l^n S + update_scale sum_j l^(n-1-j+e) y_j (x) z_j
// All powers are of one head's decay and not above 1 where it decays, so nothing has to be scaled back.
//
// A workgroup of four wavefronts holds 64 NV columns of one head's state in registers, 16 NV a wavefront, as the tiles of a
// matrix product: they are the left operand of x S as they lie.  x, y and z of a chunk are staged in LDS, the next chunk's loads
// stay in flight in registers meanwhile.  Each wavefront works out the whole triangle x_i . y_j by itself: its tiles, too, are an
// operand as they lie, and a second barrier a chunk would cost more than the products.  Output tiles are taken as their
// transpose, in which a lane holds neighbouring columns of one token.
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

constexpr int kChunkThreads = 256;

// The pieces along time that different workgroups take (A.T tokens from place `segment * segment_tokens` on)
struct ChunkArgs {
    AttentionArgs a;
    int64_t segment_tokens;     // a multiple of the chunk; at least T where there is one segment
    int segments;
    float *states;              // [segments][B][heads][rows][columns]: state-only launches write a segment's own, others read what lies before it
};

// A tile of C tokens x W values: global memory -> registers -> LDS (E), zeros where there is nothing.  The loads are
// unconditional (what is not there is read from the first token instead, and dropped on the way to LDS), so that all are in flight at once.
template <typename T, typename E, int C, int W>
struct TileLoader {
    static constexpr int GROUP = 16 / (sizeof(T) > sizeof(E) ? sizeof(T) : sizeof(E));      // values of a load
    static constexpr int ROW = W / GROUP, COUNT = C * ROW / kChunkThreads;
    static_assert(C * ROW % kChunkThreads == 0);
    Pack<T, GROUP> held[COUNT];

    static __device__ bool there(int i, int n, int width, int *r, int *c)
    {
        const int at = threadIdx.x + i * kChunkThreads;
        *r = at / ROW;
        *c = at % ROW * GROUP;
        return *r < n && *c + GROUP <= width;
    }
    // token r of the tile is at p + r * stride; 1 <= n of them are there, `width` values each
    __device__ void load(const T *p, int64_t stride, int n, int width)
    {
        if (width < GROUP) return;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            int r, c;
            const bool ok = there(i, n, width, &r, &c);
            held[i] = *(const Pack<T, GROUP> *)(p + (ok ? r * stride + c : 0));
        }
    }
    __device__ void store(E *tile, int pitch, const T *p, int64_t stride, int n, int width) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            int r, c;
            const bool ok = there(i, n, width, &r, &c);
            struct alignas(GROUP * sizeof(E)) { E v[GROUP]; } row;
#pragma unroll
            for (int j = 0; j < GROUP; ++j) row.v[j] = ok ? (E)held[i].v[j] : (E)0.0f;
            *(decltype(row) *)(tile + r * pitch + c) = row;
        }
        // the last values of rows that are no whole number of groups (after the zeros of the same thread)
        if (width < W && width % GROUP)
#pragma unroll 1
            for (int i = 0; i < COUNT; ++i) {
                const int at = threadIdx.x + i * kChunkThreads, r = at / ROW, c = at % ROW * GROUP;
                if (r < n && c < width && c + GROUP > width)
#pragma unroll 1
                    for (int j = c; j < width; ++j) tile[r * pitch + j] = (E)p[r * stride + j];
            }
    }
};

// Column of the state that line r of tile `tile` of a wavefront's NV tiles stands for: two tiles of 16-bit outputs alternate in groups of
// four, so that a lane's values of both are eight neighbours (a 16-byte store)
template <typename O, int NV>
__device__ inline int chunk_column(int tile, int r)
{
    return sizeof(O) == 2 && NV == 2 ? r / 4 * 8 + tile * 4 + r % 4 : tile * 16 + r;
}

// One token after the other, for the chunk in LDS (see above).  store(r, nv, o_r at the column of line `line`)
template <bool OUTPUT, int KT, int NV, typename E, typename Column, typename Store>
__device__ inline void chunk_by_token(const AttentionArgs &A, float g, int n, const E *xs, const E *ys, int kpitch, const E *zs, int vpitch,
                                            f4 (&s)[KT][NV], Column column, Store store)
{
    const int quad = threadIdx.x % 64 / 16;
    const float shrink = expm1f(g);
    for (int r = 0; r < n; ++r) {
#pragma unroll
        for (int nv = 0; nv < NV; ++nv) {
            const float z = A.update_scale * (float)zs[r * vpitch + column(nv)];
            float part = 0.0f;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * kt + 4 * quad + i;
                    if (row >= A.rows) continue;
                    float c = s[kt][nv][i];
                    if (!A.reversed) c = fmaf(c, shrink, c);
                    c = fmaf((float)ys[r * kpitch + row], z, c);
                    if (OUTPUT) part = fmaf((float)xs[r * kpitch + row], c, part);
                    if (A.reversed) c = fmaf(c, shrink, c);
                    s[kt][nv][i] = c;
                }
            if (OUTPUT) {
                part += __shfl_xor(part, 16);
                part += __shfl_xor(part, 32);
                store(r, nv, A.out_scale * part);
            }
        }
    }
}

// T, O: types of operands and output; E: type in LDS; K: rows of the state, rounded up; PARTS: fragments that the state's update takes
// each weighted z in (Matrix<E>::EXACT: all its digits); OUTPUT: 0 for launches that only work out the segments' own states
template <typename T, typename O, typename E, int C, int K, int NV, int PARTS, bool OUTPUT, int WAVES>
__global__ __launch_bounds__(kChunkThreads, WAVES) void sig_attention_chunk_kernel(ChunkArgs G)
{
    using M = Matrix<E>;
    using Frag = typename M::Frag;
    constexpr int VT = 64 * NV, KPITCH = K + M::PAD, VPITCH = VT + M::PAD;
    constexpr int MT = C / 16, STEPS = C / M::STEP, KSTEPS = K / M::STEP, SUB = M::SUB;
    constexpr int SPLIT = SUB == 2 ? 2 : 1;       // bfloat16 fragments of the state and of the triangle: 16 digits
    const AttentionArgs &A = G.a;
    __shared__ __attribute__((aligned(16))) E xs[OUTPUT ? C * KPITCH : 8], ys[C * KPITCH], zs[C * VPITCH];
    __shared__ float power[C + 1];                // l^0 .. l^C

    const int64_t head = blockIdx.x % A.heads, b = blockIdx.x / A.heads;
    const int lane = threadIdx.x % 64, line = lane % 16, quad = lane / 16, wave = threadIdx.x / 64;
    const int c0 = blockIdx.y * VT;               // first column of the workgroup, and of the wavefront in it
    const int wave_column = wave * 16 * NV;
    const int64_t length = attention_length(A, b), first = (int64_t)blockIdx.z * G.segment_tokens;
    const int64_t last = first + G.segment_tokens < length && (int)blockIdx.z + 1 < G.segments ? first + G.segment_tokens : length;
    const float g = A.log_decay[head];
    for (int i = threadIdx.x; i <= C; i += kChunkThreads) power[i] = i == 0 ? 1.0f : expf((float)i * g);

    // token number i of the pass is at x + i * stride
    const int64_t start = A.reversed ? length - 1 : 0;
    const int64_t xstep = A.reversed ? -A.xs[1] : A.xs[1], ystep = A.reversed ? -A.ys[1] : A.ys[1];
    const int64_t zstep = A.reversed ? -A.zs[1] : A.zs[1], ostep = A.reversed ? -A.os[1] : A.os[1];
    const T *x = (const T *)A.x + b * A.xs[0] + head / A.x_group * A.xs[2] + start * A.xs[1];
    const T *y = (const T *)A.y + b * A.ys[0] + head / A.y_group * A.ys[2] + start * A.ys[1];
    const T *z = (const T *)A.z + b * A.zs[0] + head / A.z_group * A.zs[2] + start * A.zs[1] + c0;
    O *o = (O *)A.o + b * A.os[0] + head * A.os[2] + start * A.os[1] + c0;

    const int width = A.columns - c0;
    auto column = [&](int nv) { return wave_column + chunk_column<O, NV>(nv, line); };
    // the state: tile (kt, nv) holds, in a lane, column `line` of the tile at rows 16 kt + 4 quad + 0..3
    f4 s[K / 16][NV];
    const int64_t head_state = (int64_t)A.rows * A.columns, at_head = (int64_t)b * A.heads + head;
    const bool own = !OUTPUT || G.segments > 1;   // states in scratch
    const int64_t row_stride = own ? A.columns : A.row_stride, column_stride = own ? 1 : A.column_stride;
    float *at_segment = G.states + ((int64_t)blockIdx.z * A.B * A.heads + at_head) * head_state;
    const float *from = !OUTPUT ? nullptr : own ? at_segment : A.state ? A.state + at_head * head_state : nullptr;
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
        for (int nv = 0; nv < NV; ++nv)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + 4 * quad + i;
                s[kt][nv][i] = from && row < A.rows && column(nv) < width ? from[row * row_stride + (c0 + column(nv)) * column_stride] : 0.0f;
            }

    TileLoader<T, E, C, K> xl, yl;
    TileLoader<T, E, C, VT> zl;
    auto load = [&](int64_t t) {
        const int n = last - t < C ? (int)(last - t) : C;
        if (OUTPUT) xl.load(x + t * xstep, xstep, n, A.rows);
        yl.load(y + t * ystep, ystep, n, A.rows);
        zl.load(z + t * zstep, zstep, n, width);
    };
    if (first < last) load(first);
    __syncthreads();
    // weights of the triangle: l^(16 d + line - 4 quad - i) for tiles d apart, nothing above the diagonal
    f4 inside[OUTPUT ? MT : 1];
    if (OUTPUT)
#pragma unroll
        for (int d = 0; d < MT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int gap = 16 * d + line - 4 * quad - i;
                inside[d][i] = gap >= 0 ? A.out_scale * A.update_scale * power[gap] : 0.0f;
            }

    bool by_token = false;
    for (int64_t t0 = first; t0 < last; t0 += C) {
        const int n = last - t0 < C ? (int)(last - t0) : C;
        if (OUTPUT) xl.store(xs, KPITCH, x + t0 * xstep, xstep, n, A.rows);
        yl.store(ys, KPITCH, y + t0 * ystep, ystep, n, A.rows);
        zl.store(zs, VPITCH, z + t0 * zstep, zstep, n, width);
        __syncthreads();
        if (t0 + C < last) load(t0 + C);

        if constexpr (!OUTPUT) {
            if (by_token) {
                chunk_by_token<false>(A, g, n, xs, ys, KPITCH, zs, VPITCH, s, column, [](int, int, float) {});
                __syncthreads();
                continue;
            }
        }
        Frag zf[STEPS][NV];
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int nv = 0; nv < NV; ++nv)
                zf[st][nv] = M::along_columns(zs + wave_column, VPITCH, st * M::STEP, [&](int r) { return chunk_column<O, NV>(nv, r); });

        if constexpr (OUTPUT) {
            f4 out[MT][NV] = {};
            // what lies before the chunk
#pragma unroll
            for (int kk = 0; kk < KSTEPS; ++kk) {
                Frag sf[NV][SPLIT];
#pragma unroll
                for (int nv = 0; nv < NV; ++nv) {
                    float values[4 * SUB];
#pragma unroll
                    for (int e = 0; e < 4 * SUB; ++e) values[e] = s[kk * SUB + e / 4][nv][e % 4];
                    M::template split<SPLIT>(values, sf[nv]);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const Frag xf = M::along_rows(xs, KPITCH, 16 * m, kk * M::STEP);
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                        for (int p = 0; p < SPLIT; ++p) out[m][nv] = M::multiply(sf[nv][p], xf, out[m][nv]);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float w = A.out_scale * power[16 * m + line + 1 - A.reversed];
#pragma unroll
                for (int nv = 0; nv < NV; ++nv) out[m][nv] *= w;
            }
            // the triangle
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                Frag xf[KSTEPS];
#pragma unroll
                for (int kk = 0; kk < KSTEPS; ++kk) xf[kk] = M::along_rows(xs, KPITCH, 16 * m, kk * M::STEP);
#pragma unroll
                for (int st = 0; st * SUB <= m; ++st) {
                    float values[4 * SUB];
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) {
                        const int j = st * SUB + sub;
                        f4 dots = {};
                        if (j <= m) {
#pragma unroll
                            for (int kk = 0; kk < KSTEPS; ++kk) dots = M::multiply(M::along_rows(ys, KPITCH, 16 * j, kk * M::STEP), xf[kk], dots);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // (a token that is not there, or comes later, must not spoil the sum with 0 * infinity)
                            const float w = j <= m ? inside[j <= m ? m - j : 0][i] : 0.0f;
                            values[4 * sub + i] = j < m || (j == m && 4 * quad + i <= line) ? w * dots[i] : 0.0f;
                        }
                    }
                    Frag pf[SPLIT];
                    M::template split<SPLIT>(values, pf);
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                        for (int p = 0; p < SPLIT; ++p) out[m][nv] = M::multiply(zf[st][nv], pf[p], out[m][nv]);
                }
            }
            float worst = 0.0f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                    for (int i = 0; i < 4; ++i) worst = fmaf(out[m][nv][i], 0.0f, worst);     // a NaN from anything that is not finite
            if (__any(!(worst == 0.0f))) {
                chunk_by_token<true>(A, g, n, xs, ys, KPITCH, zs, VPITCH, s, column, [&](int r, int nv, float value) {
                    if (quad == 0 && column(nv) < width) o[(t0 + r) * ostep + column(nv)] = from_float<O>(value);
                });
                __syncthreads();
                continue;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int r = 16 * m + line;
                if (r >= n) continue;
                O *to = o + (t0 + r) * ostep;
                constexpr int RUN = sizeof(O) == 2 && NV == 2 ? 8 : 4;
#pragma unroll
                for (int q = 0; q < 4 * NV / RUN; ++q) {
                    const int at = wave_column + (RUN == 8 ? 8 * quad : 16 * q + 4 * quad);
                    Pack<O, RUN> values;
#pragma unroll
                    for (int j = 0; j < RUN; ++j) values.v[j] = from_float<O>(out[m][RUN == 8 ? j / 4 : q][j % 4]);
                    if (at + RUN <= width) {
                        *(Pack<O, RUN> *)(to + at) = values;
                    } else {
#pragma unroll
                        for (int j = 0; j < RUN; ++j)
                            if (at + j < width) to[at + j] = values.v[j];
                    }
                }
            }
        }

        // the state behind the chunk.  l^n = 1 + (l^n - 1): the power itself, rounded, would drift over many chunks where little decays
        const float shrink = expm1f((float)n * g);
#pragma unroll
        for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
            for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kt][nv][i] = fmaf(s[kt][nv][i], shrink, s[kt][nv][i]);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            Frag wf[NV][PARTS];
#pragma unroll
            for (int nv = 0; nv < NV; ++nv) {
                float values[4 * SUB];
#pragma unroll
                for (int e = 0; e < 4 * SUB; ++e) {
                    const int j = st * M::STEP + e / 4 * 16 + 4 * quad + e % 4, ahead = n - 1 - j + A.reversed;
                    values[e] = ahead >= 0 ? M::value(zf[st][nv], e) * (A.update_scale * power[ahead]) : 0.0f;
                }
                M::template split<PARTS>(values, wf[nv]);
            }
#pragma unroll
            for (int kt = 0; kt < K / 16; ++kt) {
                const Frag yf = M::along_columns(ys, KPITCH, st * M::STEP, [&](int r) { return 16 * kt + r; });
#pragma unroll
                for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) s[kt][nv] = M::multiply(yf, wf[nv][p], s[kt][nv]);
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
                    for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                        for (int i = 0; i < 4; ++i) worst = fmaf(s[kt][nv][i], 0.0f, worst);
            if (__syncthreads_or(!(worst == 0.0f))) {
                by_token = true;
#pragma unroll
                for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv) s[kt][nv] = f4{};
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
            for (int64_t i = threadIdx.x; i < (A.T - length) * left; i += kChunkThreads) rest[(length + i / left) * A.os[1] + i % left] = from_float<O>(0.0f);
        }
        if (own || !A.state_out) return;
    }
    float *to = own ? at_segment : A.state_out + at_head * head_state;
#pragma unroll
    for (int kt = 0; kt < K / 16; ++kt)
#pragma unroll
        for (int nv = 0; nv < NV; ++nv)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * kt + 4 * quad + i;
                if (row < A.rows && column(nv) < width) to[row * row_stride + (c0 + column(nv)) * column_stride] = s[kt][nv][i];
            }
}

// The instance for `G`: columns of a workgroup 64 nv; rows up to 256
template <typename T, typename O, typename E, int C, int PARTS, bool OUTPUT>
void launch_chunk_instance(const ChunkArgs &G, int nv, hipStream_t st)
{
    const AttentionArgs &A = G.a;
    const dim3 grid((unsigned)(A.B * A.heads), (unsigned)((A.columns + 64 * nv - 1) / (64 * nv)), (unsigned)G.segments);
    auto go = [&](auto k) {
        constexpr int K = decltype(k)::value;
        constexpr int TOKENS = K > 192 && C > 32 ? 32 : C, WIDE = K <= 128 ? 2 : 1;      // (registers)
        if (WIDE == 2 && nv == 2) sig_attention_chunk_kernel<T, O, E, TOKENS, K, WIDE, PARTS, OUTPUT, K * WIDE <= 64 ? 2 : 1><<<grid, kChunkThreads, 0, st>>>(G);
        else sig_attention_chunk_kernel<T, O, E, TOKENS, K, 1, PARTS, OUTPUT, K <= 64 ? 2 : 1><<<grid, kChunkThreads, 0, st>>>(G);
    };
    if (A.rows <= 32) go(std::integral_constant<int, 32>());
    else if (A.rows <= 64) go(std::integral_constant<int, 64>());
    else if (A.rows <= 128) go(std::integral_constant<int, 128>());
    else if (A.rows <= 192) go(std::integral_constant<int, 192>());
    else go(std::integral_constant<int, 256>());
}

template <typename T, typename E, int C>
void launch_chunk(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st)
{
    constexpr int PARTS = Matrix<E>::EXACT;
    if (!output) launch_chunk_instance<T, T, E, C, PARTS, false>(G, nv, st);
    else if (partial) launch_chunk_instance<T, float, E, C, PARTS, true>(G, nv, st);
    else launch_chunk_instance<T, T, E, C, PARTS, true>(G, nv, st);
}

// one for each type of the operands, in a file of its own; partial: float32 output
void launch_chunk_f32(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st);
void launch_chunk_bf16(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st);
void launch_chunk_f16(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st);

}  // namespace sig
#endif
