// Linear attention on matrix instructions, C tokens at a time (sig_attention.h).
//
// With j, i the places of two tokens in a chunk of n tokens (n = C but for the last one), S the state in front of it, and e = 1 for a
// reversed pass, which decays behind a token, else 0:
//   o_i = out_scale l^(i+1-e) x_i S + out_scale update_scale sum_{j <= i} l^(i-j) (x_i . y_j) z_j
//   S  <- l^n S + update_scale sum_j l^(n-1-j+e) y_j (x) z_j
// All powers are of one head's decay and not above 1 where it decays, so nothing has to be scaled back.
//
// A workgroup of four wavefronts holds 64 NV columns of one head's state in registers, 16 NV a wavefront, as the tiles of a matrix
// product: they are the left operand of x S as they lie.  x, y and z of a chunk are staged in LDS, the next chunk's loads stay in flight in registers
// meanwhile.  The tiles of the triangle are shared out over the wavefronts and passed on through LDS, as the fragments that
// everyone reads.  Output tiles are taken as their transpose, in which a lane holds neighbouring columns of one token.
//
// Bound by neither memory nor the matrix units, but by what a chunk's steps wait for one after the other (operands from LDS, barriers) on the
// two workgroups that a unit holds.  Measured, on two cards: 65,536 tokens, 8 heads of 128 x 128 bfloat16, 234 and 243 us (2.2 TB/s of what goes in and
// out; matrix units busy for 29% of the main launch, vector instructions 40%); 8 x 4,096 tokens, 16 heads, training, 688 and 714 us; 64 x 255
// tokens, 4 heads of 64 x 64 float32, 26 us (2.6 TB/s).  Chunks of 64 tokens of bfloat16, since each also rounds the state anew for its
// products (32 tokens take as long: that batch 0.99 times, 64 sequences of 3,000 tokens 1.015), but 32 where the state has 256 rows (LDS then holds two
// workgroups) or sequences are short; 32 of float32.
//
// A product of matrices multiplies every pair: 0 x infinity where the triangle is empty, and the parts of an infinite number.  A chunk
// whose output is not finite is therefore worked out again token by token, by the wavefronts of those columns, so that what is not a number
// reaches what it reaches in the recurrence.  Behind it chunks go on as chunks, unless something in the state is not finite: that lasts, and
// the rest of the segment goes token by token (8 x 4,096 tokens, 16 heads of 128 x 128 bfloat16, forward: an infinite query in each 619 us, an infinite
// key 11.5 ms, neither 235).  Launches without output: the whole segment, if its state is not finite.
#ifndef SIG_ATTENTION_CHUNK_H
#define SIG_ATTENTION_CHUNK_H

#include <type_traits>

#include "sig_attention.h"
#include "sig_matrix.h"

namespace sig {

constexpr int kChunkThreads = 256;

template <int N>
using Number = std::integral_constant<int, N>;

constexpr int kMostPasses = 3;

// Passes of the same batch, heads and rows that one launch takes, and the segments along time that different workgroups take: A.T
// tokens from place segment * segment_tokens on
struct ChunkArgs {
    AttentionArgs a[kMostPasses];
    int passes, segments;
    int64_t segment_tokens;     // a multiple of the chunk; at least T where there is one segment
    int64_t states_apart;       // floats of `states` between passes
    // [passes][segments][B][heads][rows][columns]: segments' own states, then what lies before the next segment; in the last place, where
    // the last segment's workgroups write over the initial state, a copy of it for the first one's
    float *states;
};

// Tiles of C tokens x W values, one after the other: global memory -> registers -> LDS (E), zeros where there is nothing.  A thread
// takes the same group of values of every ROWS-th token.  Its loads are unconditional (what is not there is read from a value
// that is, and dropped on the way to LDS), so that all are in flight at once.
template <typename T, typename E, int C, int W, int THREADS>
struct TileLoader {
    static constexpr int GROUP = 16 / (sizeof(T) > sizeof(E) ? sizeof(T) : sizeof(E));      // values of a load
    static constexpr int WIDE = W <= 32 ? 32 : W <= 64 ? 64 : W <= 128 ? 128 : 256;         // (threads beyond W load and drop)
    static constexpr int ROWS = THREADS / (WIDE / GROUP), COUNT = C / ROWS;
    static_assert(THREADS % (WIDE / GROUP) == 0 && C % ROWS == 0);
    const T *p;          // of the next tile
    int64_t stride;      // between tokens
    int width;           // values of a token
    struct Tile { Pack<T, GROUP> held[COUNT]; };      // a thread's part, on its way

    static __device__ int row_of(int thread) { return thread / (WIDE / GROUP); }
    static __device__ int place_of(int thread) { return thread % (WIDE / GROUP) * GROUP; }

    // token 0 of the first tile is at `tokens`
    __device__ TileLoader(const T *tokens, int64_t stride_, int width_) : stride(stride_), width(width_)
    {
        const int row = row_of(threadIdx.x), place = place_of(threadIdx.x);
        p = tokens + row * stride + (place + GROUP <= width ? place : 0);
    }
    // the next tile, of which 1 <= n <= C tokens are there; thread: threadIdx.x
    __device__ void load(Tile &tile, int n, int thread)
    {
        int values = width;
        asm volatile("" : "+s"(values));      // (compared anew: the answer would be kept in a register of every lane)
        if (values >= GROUP) {
            if (n == C) {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) tile.held[i] = *(const Pack<T, GROUP> *)(p + i * ROWS * stride);
            } else {
#pragma unroll
                for (int i = 0; i < COUNT; ++i) {
                    const int r = row_of(thread) + i * ROWS;
                    tile.held[i] = *(const Pack<T, GROUP> *)(p + ((r < n ? r : n - 1) - row_of(thread)) * stride);
                }
            }
        }
        p += C * stride;
    }
    // the last tile again
    __device__ void back() { p -= C * stride; }
    // the tile of the last load(from, n, thread)
    __device__ void store(const Tile &from, E *tile, int pitch, int n, int thread) const
    {
        const int row = row_of(thread), place = place_of(thread);
        const bool there = place + GROUP <= width;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int r = row + i * ROWS;
            const bool ok = there && r < n;
            struct { E v[GROUP]; } values;
#pragma unroll
            for (int j = 0; j < GROUP; ++j) values.v[j] = (E)from.held[i].v[j];
            using u4 = __attribute__((ext_vector_type(4))) unsigned;
            u4 bits = __builtin_bit_cast(u4, values);
            bits = ok ? bits : u4{};
            if (W == WIDE || place < W) *(u4 *)(tile + r * pitch + place) = bits;
        }
        // the last values of tokens that are no whole number of groups (after the zeros of the same thread, which then reads from place 0)
        const int rest = width % GROUP, c = place;
        if (width < W && rest && c < width && c + GROUP > width) {
            const T *last = p - C * stride + c;
#pragma unroll 1
            for (int r = row; r < n; r += ROWS, last += ROWS * stride)
#pragma unroll 1
                for (int j = 0; j < rest; ++j) tile[r * pitch + c + j] = (E)last[j];
        }
    }
};

// One token after the other, for the chunk in LDS (see above).  store(r, nv, o_r at the lane's column of tile nv)
template <bool OUTPUT, int KT, int NV, typename E, typename Row, typename Store>
__device__ inline void chunk_by_token(const AttentionArgs &A, float g, int n, const E *xs, int xpitch, const E *ys, int ypitch, const E *zs, int zpitch,
                                      f4 (&s)[KT][NV], int first_row, Row row_of, int column, Store store)
{
    const Decay decay(g, 1.0f);
#pragma unroll 1
    for (int r = 0; r < n; ++r) {
        int rows = A.rows;
        asm volatile("" : "+v"(rows));      // (compared anew: the masks of all rows would not fit the scalar registers)
#pragma unroll
        for (int nv = 0; nv < NV; ++nv) {
            const float z = A.update_scale * (float)zs[r * zpitch + column + 16 * nv];
            float part = 0.0f;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = first_row + row_of(kt) + i;
                    if (row >= rows) continue;
                    float c = s[kt][nv][i];
                    if (!A.reversed) c = decay(c);
                    c = fmaf((float)ys[r * ypitch + row], z, c);
                    if (OUTPUT) part = fmaf((float)xs[r * xpitch + row], c, part);
                    if (A.reversed) c = decay(c);
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

// The order of what has been written since the last call: LOADS reads of LDS, then PRODUCTS products with vector instructions between them
template <int LOADS, int PRODUCTS>
__device__ inline void interleave()
{
    __builtin_amdgcn_sched_group_barrier(0x100, LOADS, 0);
#pragma unroll
    for (int i = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// T, O: types of operands and output; E: type in LDS; K: rows of the state, rounded up; NV: tiles of 16 columns a wavefront; OUTPUT: 0 for launches that
// only work out the segments' own states
// Two workgroups a unit, where LDS has room for them (with one, whose registers the compiler then spreads out: 192 rows of bfloat16 1.15 to 1.6
// times as long, 192 and 256 rows of float32 1.1 to 1.3).
template <typename T, typename O, typename E, int C, int K, int NV, bool OUTPUT>
__global__ __launch_bounds__(kChunkThreads, C == 32 || K <= 192 ? 2 : 1) void sig_attention_chunk_kernel(ChunkArgs G)
{
    using M = Matrix<E>;
    using Frag = typename M::Frag;
    constexpr int THREADS = kChunkThreads, WAVES = THREADS / 64, VT = 64 * NV;
    constexpr int XPITCH = K + M::PAD, YPITCH = K + M::COLUMN_PAD, ZPITCH = VT + M::COLUMN_PAD;
    constexpr int MT = C / 16, STEPS = C / M::STEP, KSTEPS = K / M::STEP, KT = K / 16, SUB = M::SUB;
    // The state itself keeps all digits of float32: each weighted z goes into its update as fragments that add up to it.  As operands of the
    // outputs' products the state and the triangle of pairs are two bfloat16 fragments, 16 digits, where those outputs are rounded to 8 (24 digits
    // leave the same errors: 65,536 tokens, 8 heads of 128 x 128, 258 us instead of 239; a training batch 792 instead of 714.  With two fragments of
    // each weighted z the batch took 673, but the gradients' state then had 16 digits too).
    constexpr int PARTS = M::EXACT, SPLIT = SUB == 2 ? 2 : 1;
    constexpr int YB = KT % 4 == 0 ? 4 : KT % 3 == 0 ? 3 : KT;      // tiles of the state whose operands are loaded at once
    const int pass = blockIdx.z % G.passes, segment = blockIdx.z / G.passes;
    const AttentionArgs &A = G.a[pass];
    if ((int)blockIdx.y * VT >= A.columns) return;
    __shared__ __attribute__((aligned(16))) E xs[OUTPUT ? C * XPITCH : 8], ys[C * YPITCH], zs[C * ZPITCH];
    __shared__ Frag triangle[OUTPUT ? MT * STEPS * SPLIT * 64 : 1];
    __shared__ int spoilt, lasting;               // whether a wavefront has met what is not finite in a chunk, and in the state
    __shared__ float after[C + 2];                // out_scale l^(i+1)
    __shared__ float gap_weight[C + 16];          // out_scale update_scale l^(i-15), zeros up to i = 14
    __shared__ float left_weight[2 * C];          // update_scale l^(C-1-i+e), zeros from i = C on

    const int64_t head = blockIdx.x % A.heads, b = blockIdx.x / A.heads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int c0 = blockIdx.y * VT, width = A.columns - c0;
    const int64_t length = attention_length(A, b), first = segment * G.segment_tokens;
    const int64_t last = first + G.segment_tokens < length && segment + 1 < G.segments ? first + G.segment_tokens : length;
    const float g = A.log_decay[head];
    if (threadIdx.x == 0) spoilt = lasting = 0;
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

    // The state: tile (kt, nv) holds, in a lane, its column at rows first_row + row_of(kt) + 0..3.  Each part of the kernel works its places out
    // anew, from a lane's number that the compiler takes for another one each time: it would keep them, and what follows from them, in registers
    // that the loop over chunks does not have.
    struct Place {
        int lane, thread, line, quad, first_row, column;      // the last four of the lane's tiles, the column in the workgroup's

        __device__ explicit Place(int wave)
        {
            int all = -1;
            asm volatile("" : "+s"(all));
            lane = __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0));
            thread = 64 * wave + lane;
            line = lane % 16;
            quad = lane / 16;
            first_row = 4 * SUB * quad;
            column = wave * 16 * NV + line;
        }
    };
    const auto row_of = [](int kt) { return kt / SUB * M::STEP + 4 * (kt % SUB); };
    f4 s[KT][NV];
    const int64_t head_state = (int64_t)A.rows * A.columns, at_head = (int64_t)b * A.heads + head;
    // A segment's state is kept behind it, and what lies before it where the last one's was.
    float *kept = G.states + pass * G.states_apart + (segment * A.B * A.heads + at_head) * head_state;
    const bool copied = segment == 0 && G.segments > 1 && A.state && A.state == A.state_out, own = segment > 0 || copied;
    const float *from = own ? kept + (copied ? G.segments - 1 : -1) * A.B * A.heads * head_state : A.state ? A.state + at_head * head_state : nullptr;
    float *state_to = !OUTPUT ? kept : segment + 1 == G.segments && A.state_out ? A.state_out + at_head * head_state : nullptr;
    const Place before(wave);
#pragma unroll
    for (int nv = 0; nv < NV; ++nv) {
        if constexpr (!OUTPUT) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) s[kt][nv] = f4{};
        } else {
            const int64_t row_stride = own ? A.columns : A.row_stride, column_stride = own ? 1 : A.column_stride;
            const float *at = from + before.first_row * row_stride + (c0 + before.column + 16 * nv) * column_stride;
            int rows = from && before.column + 16 * nv < width ? A.rows - before.first_row : 0;
            asm volatile("" : "+v"(rows));
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kt][nv][i] = row_of(kt) + i < rows ? at[(row_of(kt) + i) * row_stride] : 0.0f;
        }
    }

    TileLoader<T, E, C, K, THREADS> xl(x + first * xstep, xstep, A.rows), yl(y + first * ystep, ystep, A.rows);
    TileLoader<T, E, C, VT, THREADS> zl(z + first * zstep, zstep, width);
    using StateTile = typename TileLoader<T, E, C, K, THREADS>::Tile;
    using ValueTile = typename TileLoader<T, E, C, VT, THREADS>::Tile;
    auto load = [&](StateTile &xt, StateTile &yt, ValueTile &zt, int64_t t, int thread) {
        const int n = last - t < C ? (int)(last - t) : C;
        if (OUTPUT) xl.load(xt, n, thread);
        yl.load(yt, n, thread);
        zl.load(zt, n, thread);
    };
    auto store = [&](const StateTile &xt, const StateTile &yt, const ValueTile &zt, int n, int thread) {
        if (OUTPUT) xl.store(xt, xs, XPITCH, n, thread);
        yl.store(yt, ys, YPITCH, n, thread);
        zl.store(zt, zs, ZPITCH, n, thread);
    };
    __syncthreads();

    // Loads from LDS are issued a block of products ahead (left alone, the compiler waits for each in turn), and the splitting of the
    // next operand goes between the products: a product keeps its unit busy for four vector instructions.
    int64_t t0 = first;
    bool again = false;          // OUTPUT: whether this wavefront still owes the chunk in LDS
    const auto lasts = [&] {      // whether something in the workgroup's state is not finite
        float worst = 0.0f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                for (int i = 0; i < 4; ++i) worst = fmaf(s[kt][nv][i], 0.0f, worst);
        if (__any(!(worst == 0.0f))) lasting = 1;
        __syncthreads();
        return lasting != 0;
    };
    while (true) {
        const Place place(wave);
        const int line = place.line, quad = place.quad, lane = place.lane;
        O *to = o + (t0 + line) * ostep + wave * 16 * NV + 4 * quad;      // the lane's outputs of the next chunk
        StateTile xt = {}, yt = {};      // (or what an earlier turn left there would be kept through all of it)
        ValueTile zt = {};
        if (t0 < last) load(xt, yt, zt, t0, place.thread);
        for (; t0 < last; t0 += C) {
            const int n = last - t0 < C ? (int)(last - t0) : C;
            store(xt, yt, zt, n, place.thread);
            __syncthreads();
            if (t0 + C < last) load(xt, yt, zt, t0 + C, place.thread);

            O *to_chunk = to;
            to += C * ostep;
            f4 out[OUTPUT ? MT : 1][NV] = {};
            Frag zf[STEPS][NV];
            if constexpr (OUTPUT) {
                // this wavefront's tiles of the triangle: tokens 16 m + line against 16 j + 4 quad + 0..3
                for (int tile = wave; tile < MT * (MT + 1) / 2; tile += WAVES) {
                    const int m = (int)(0x3333222110ull >> 4 * tile & 15), j = tile - m * (m + 1) / 2;
                    f4 dots = {};
                    float weight[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) weight[i] = gap_weight[15 + 16 * (m - j) + line - 4 * quad - i];
                    constexpr int TB = KSTEPS < 4 ? KSTEPS : 4;
#pragma unroll
                    for (int k0 = 0; k0 < KSTEPS; k0 += TB) {
                        Frag left[TB], right[TB];
#pragma unroll
                        for (int kk = 0; kk < TB && k0 + kk < KSTEPS; ++kk) {
                            left[kk] = M::along_rows(lane, ys, YPITCH, 16 * j, (k0 + kk) * M::STEP);
                            right[kk] = M::along_rows(lane, xs, XPITCH, 16 * m, (k0 + kk) * M::STEP);
                        }
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int kk = 0; kk < TB && k0 + kk < KSTEPS; ++kk) dots = M::multiply(left[kk], right[kk], dots);
                    }
                    float values[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) values[i] = j < m || 4 * quad + i <= line ? weight[i] * dots[i] : 0.0f;      // (a later token may be infinite)
                    M::template put<SPLIT>(values, triangle + (m * STEPS + j / SUB) * SPLIT * 64 + lane, j % SUB);
                }
                // what lies before the chunk
                Frag xf[2][MT], sf[2][SPLIT];
                auto state_step = [&](int kk, int nv, Frag (&to)[SPLIT]) {
                    float values[4 * SUB];
#pragma unroll
                    for (int e = 0; e < 4 * SUB; ++e) values[e] = s[kk * SUB + e / 4][nv][e % 4];
                    M::template split<SPLIT>(values, to);
                };
#pragma unroll
                for (int m = 0; m < MT; ++m) xf[0][m] = M::along_rows(lane, xs, XPITCH, 16 * m, 0);
                state_step(0, 0, sf[0]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kk = 0; kk < KSTEPS; ++kk)
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv) {
                        const int now = (kk * NV + nv) % 2;
                        if (nv == 0 && kk + 1 < KSTEPS) {
#pragma unroll
                            for (int m = 0; m < MT; ++m) xf[(kk + 1) % 2][m] = M::along_rows(lane, xs, XPITCH, 16 * m, (kk + 1) * M::STEP);
                        } else if (nv == NV - 1 && kk + 1 == KSTEPS) {
#pragma unroll
                            for (int st = 0; st < STEPS; ++st)
#pragma unroll
                                for (int i = 0; i < NV; ++i) zf[st][i] = M::template along_columns<false>(lane, zs, ZPITCH, st * M::STEP, wave * 16 * NV + 16 * i);
                        }
                        if (nv + 1 < NV) state_step(kk, nv + 1, sf[1 - now]);
                        else if (kk + 1 < KSTEPS) state_step(kk + 1, 0, sf[1 - now]);
#pragma unroll
                        for (int p = 0; p < SPLIT; ++p)
#pragma unroll
                            for (int m = 0; m < MT; ++m) out[m][nv] = M::multiply(sf[now][p], xf[kk % 2][m], out[m][nv]);
                        interleave<MT, SPLIT * MT * M::PRODUCTS>();
                    }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const float w = after[16 * m + line + 1 - A.reversed];
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv) out[m][nv] *= w;
                }
                __syncthreads();
                // the triangle
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    Frag pairs[MT][SPLIT];
#pragma unroll
                    for (int m = st * SUB; m < MT; ++m)
#pragma unroll
                        for (int p = 0; p < SPLIT; ++p) pairs[m][p] = triangle[((m * STEPS + st) * SPLIT + p) * 64 + lane];
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int p = 0; p < SPLIT; ++p)
#pragma unroll
                        for (int m = st * SUB; m < MT; ++m)
#pragma unroll
                            for (int nv = 0; nv < NV; ++nv) out[m][nv] = M::multiply(zf[st][nv], pairs[m][p], out[m][nv]);
                }
                float worst = 0.0f;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                        for (int i = 0; i < 4; ++i) worst = fmaf(out[m][nv][i], 0.0f, worst);     // a NaN from anything that is not finite
                again = __any(!(worst == 0.0f));
                if (again) {
                    spoilt = 1;
                } else {
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if (16 * m + line >= n) continue;
#pragma unroll
                        for (int nv = 0; nv < NV; ++nv) {
                            O *at = to_chunk + 16 * m * ostep + 16 * nv;
                            Pack<O, 4> values;
#pragma unroll
                            for (int j = 0; j < 4; ++j) values.v[j] = from_float<O>(out[m][nv][j]);
                            const int left = width - (wave * 16 * NV + 16 * nv + 4 * quad);
                            if (left >= 4) {
                                store_pack(at, values);
                            } else {
#pragma unroll
                                for (int j = 0; j < 3; ++j)
                                    if (j < left) at[j] = values.v[j];
                            }
                        }
                    }
                }
            } else {
#pragma unroll
                for (int st = 0; st < STEPS; ++st)
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv) zf[st][nv] = M::template along_columns<false>(lane, zs, ZPITCH, st * M::STEP, wave * 16 * NV + 16 * nv);
            }
            if (!again) {
                // the state behind the chunk (a finite one; see Decay)
                const float shrink = expm1f((float)n * g);
                constexpr int BLOCKS = KT / YB, ALL = STEPS * BLOCKS;
                static_assert(KT % YB == 0);
                Frag yf[2][YB], wf[2][NV][PARTS];
                auto y_block = [&](int block, Frag (&to)[YB]) {
#pragma unroll
                    for (int i = 0; i < YB; ++i) {
                        const int kt = block % BLOCKS * YB + i;
                        to[i] = M::template along_columns<true>(lane, ys, YPITCH, block / BLOCKS * M::STEP, kt / SUB * M::STEP, kt % SUB);
                    }
                };
                auto z_step = [&](int st, Frag (&to)[NV][PARTS]) {
                    float weight[4 * SUB];
#pragma unroll
                    for (int e = 0; e < 4 * SUB; ++e) weight[e] = left_weight[C - n + st * M::STEP + e / 4 * 16 + 4 * quad + e % 4];
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv) {
                        float values[4 * SUB];
#pragma unroll
                        for (int e = 0; e < 4 * SUB; ++e) values[e] = weight[e] * M::value(zf[st][nv], e);
                        M::template split<PARTS>(values, to[nv]);
                    }
                };
                auto shrink_block = [&](int block) {
#pragma unroll
                    for (int kt = block * YB; kt < (block + 1) * YB; ++kt)
#pragma unroll
                        for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                            for (int i = 0; i < 4; ++i) s[kt][nv][i] = fmaf(s[kt][nv][i], shrink, s[kt][nv][i]);
                };
                y_block(0, yf[0]);
                shrink_block(0);
                z_step(0, wf[0]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int block = 0; block < ALL; ++block) {
                    const int st = block / BLOCKS, k0 = block % BLOCKS * YB;
                    if (block + 1 < ALL) y_block(block + 1, yf[(block + 1) % 2]);
                    if (block + 1 < BLOCKS) shrink_block(block + 1);
                    if (block % BLOCKS == BLOCKS - 1 && st + 1 < STEPS) z_step(st + 1, wf[(st + 1) % 2]);
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
#pragma unroll
                        for (int nv = 0; nv < NV; ++nv)
#pragma unroll
                            for (int i = 0; i < YB; ++i) s[k0 + i][nv] = M::multiply(yf[block % 2][i], wf[st % 2][nv][p], s[k0 + i][nv]);
                    interleave<YB * M::COLUMN_READS, PARTS * NV * YB * M::PRODUCTS>();
                }
            }
            __syncthreads();
            if (OUTPUT && spoilt) break;
        }
        if constexpr (!OUTPUT) {
            if (lasts()) {
                // the whole segment again, token by token
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int nv = 0; nv < NV; ++nv) s[kt][nv] = f4{};
                yl = TileLoader<T, E, C, K, THREADS>(y + first * ystep, ystep, A.rows);
                zl = TileLoader<T, E, C, VT, THREADS>(z + first * zstep, zstep, width);
                t0 = first - C;
            }
        } else if (t0 + C < last) {
            // (loaded anew behind the chunk in LDS: its registers are wanted)
            xl.back();
            yl.back();
            zl.back();
        }
        // Token by token: first, with output, the chunk in LDS for those who could not take it.  From there on in chunks again, unless something
        // in the state is not finite: that stays so, and so does what reads it.
        bool chunks = false;
        const Place alone(wave);
        for (; t0 < last; t0 += C) {
            const int n = last - t0 < C ? (int)(last - t0) : C;
            if (t0 >= first && (!OUTPUT || again))
                chunk_by_token<OUTPUT>(A, g, n, xs, XPITCH, ys, YPITCH, zs, ZPITCH, s, alone.first_row, row_of, alone.column, [&](int r, int nv, float value) {
                    if (alone.quad == 0 && alone.column + 16 * nv < width) o[(t0 + r) * ostep + alone.column + 16 * nv] = from_float<O>(value);
                });
            again = true;
            const bool stays = !OUTPUT || lasts();
            if (!OUTPUT) __syncthreads();
            if (t0 + C >= last) break;
            if (!stays) {
                spoilt = 0;
                again = false;
                chunks = true;
                t0 += C;
                break;
            }
            const int more = last - t0 - C < C ? (int)(last - t0 - C) : C;
            StateTile x_next = {}, y_next = {};
            ValueTile z_next = {};
            load(x_next, y_next, z_next, t0 + C, alone.thread);
            store(x_next, y_next, z_next, more, alone.thread);
            __syncthreads();
        }
        if (!chunks) break;
    }

    if constexpr (OUTPUT) {
        // behind the length: zeros, a segment's own (four columns a thread)
        const int64_t end = segment + 1 < G.segments ? first + G.segment_tokens : A.T;
        constexpr int LANES = VT / 4;
        const int thread = Place(wave).thread, c4 = thread % LANES * 4, left = width - c4;
        for (int64_t t = (first > length ? first : length) + thread / LANES; t < end; t += THREADS / LANES) {
            O *rest = (O *)A.o + b * A.os[0] + head * A.os[2] + t * A.os[1] + c0 + c4;
            if (left >= 4) {
                store_pack(rest, Pack<O, 4>{});
            } else {
                for (int j = 0; j < left; ++j) rest[j] = from_float<O>(0.0f);
            }
        }
        if (!state_to) return;
    }
    const int64_t row_stride = OUTPUT ? A.row_stride : A.columns, column_stride = OUTPUT ? A.column_stride : 1;
    const Place behind(wave);
#pragma unroll
    for (int nv = 0; nv < NV; ++nv) {
        float *to = state_to + behind.first_row * row_stride + (c0 + behind.column + 16 * nv) * column_stride;
        int rows = behind.column + 16 * nv < width ? A.rows - behind.first_row : 0;
        asm volatile("" : "+v"(rows));
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (row_of(kt) + i < rows) to[(row_of(kt) + i) * row_stride] = s[kt][nv][i];
    }
}

// Rows of the state that an instance holds, for so many: whole steps of the products (32 rows, 16 of float32), since every
// padded row costs its products.  Float32, 16 sequences of ragged length, 12 heads of 40 rows by 72 columns and the gradient:
// 503 us with 48 and 80 rows, 692 us with 64 and 128.
inline int chunk_rows(int rows, int type)
{
    const bool halves = type != SIG_BF16;
    return rows <= 32 ? 32 : halves && rows <= 48 ? 48 : rows <= 64 ? 64 : halves && rows <= 80 ? 80 : rows <= 96 ? 96 : rows <= 128 ? 128 : rows <= 192 ? 192 : 256;
}

// Up to so many tokens bfloat16 goes in chunks of 32 too (more workgroups a unit, fewer tokens to fill up).  Measured (us, chunks of 64; of 32):
//   tokens                                        16         48         96         192        256        3,000
//   128 sequences, 16 heads of 64 x 64            25; 17     26; 22     37; 27     49; 42     61; 53     754; 766
//   64 sequences, 16 heads of 128 x 128, training 90; 70     97; 98     148; 126   210; 208   283; 279   3,132; 3,178
//   4 sequences, 8 heads of 128 x 128             10; 8      10; 10     13; 11     16; 17     19; 20     65; 65
constexpr int kShortTokens = 192;

// The instance for `G`: up to 64 nv columns a workgroup
template <typename T, typename O, typename E, int C, bool OUTPUT>
void launch_chunk_instance(const ChunkArgs &G, int nv, hipStream_t st)
{
    const AttentionArgs &A = G.a[0];
    int columns = 0;
    for (int i = 0; i < G.passes; ++i) columns = G.a[i].columns > columns ? G.a[i].columns : columns;
    auto go = [&](auto k, auto n) {
        constexpr int NV = decltype(n)::value;
        const dim3 grid((unsigned)(A.B * A.heads), (unsigned)((columns + 64 * NV - 1) / (64 * NV)),
                        (unsigned)(G.passes * (OUTPUT ? G.segments : G.segments - 1)));
        constexpr int K = decltype(k)::value;
        if constexpr (OUTPUT && C == 64 && K >= 64 && K < 256) {
            if (A.T <= kShortTokens) {
                sig_attention_chunk_kernel<T, O, E, 32, K, NV, OUTPUT><<<grid, kChunkThreads, 0, st>>>(G);
                return;
            }
        }
        sig_attention_chunk_kernel<T, O, E, K == 256 ? 32 : C, K, NV, OUTPUT><<<grid, kChunkThreads, 0, st>>>(G);
    };
    constexpr int WIDE = sizeof(O) == sizeof(T) || sizeof(E) == 4 ? 2 : 1;       // (registers)
    auto either = [&](auto k) { nv == 2 ? go(k, Number<2>()) : go(k, Number<1>()); };
    switch (chunk_rows(A.rows, sizeof(E) == 2 ? SIG_BF16 : SIG_F32)) {
    case 32: either(Number<32>()); break;
    case 48: if constexpr (sizeof(E) == 4) either(Number<48>()); break;
    case 64: either(Number<64>()); break;
    case 80: if constexpr (sizeof(E) == 4) either(Number<80>()); break;
    case 96: nv == 2 ? go(Number<96>(), Number<WIDE>()) : go(Number<96>(), Number<1>()); break;
    case 128: nv == 2 ? go(Number<128>(), Number<WIDE>()) : go(Number<128>(), Number<1>()); break;
    case 192: go(Number<192>(), Number<1>()); break;
    default: go(Number<256>(), Number<1>());
    }
}

template <typename T, typename E, int C>
void launch_chunk(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st)
{
    if (!output) launch_chunk_instance<T, T, E, C, false>(G, nv, st);
    else if (partial) launch_chunk_instance<T, float, E, C, true>(G, nv, st);
    else launch_chunk_instance<T, T, E, C, true>(G, nv, st);
}

// one for each type of the operands, in a file of its own; partial: float32 output
void launch_chunk_f32(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st);
void launch_chunk_bf16(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st);
void launch_chunk_f16(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st);

}  // namespace sig
#endif
