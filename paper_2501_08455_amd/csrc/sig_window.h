// Softmax attention with a sliding window and first tokens that stay visible: kernels (include/sig_sequence.h).
//
// Token t sees token s <= t if t - s < window or s < sinks.  With z_ts = c q_t . k_s over what t sees, m_t = max z_ts and r_t = 1 / sum exp(z_ts - m_t):
//   p_ts = exp(z_ts - m_t) r_t,   o_t = sum_s p_ts v_s
// One pass over the keys: a running maximum and sum, and what is added up so far scaled down whenever the maximum grows.  The gradient works p out
// again from m and r, which the forward pass leaves.  With g the upstream gradient and D_t = g_t . o_t:
//   u_ts = p_ts (g_t . v_s - D_t),   grad q_t = c sum_s u_ts k_s,   grad k_s = c sum_t u_ts q_t,   grad v_s = sum_t p_ts g_t
//
// A wavefront holds M lines as its own operand in registers (queries; keys and values in the last kernel) and walks over tiles of the others in LDS, which
// four wavefronts share.  All products are taken with the own lines as the result's columns, so that a lane has to do with one line only:
// its maximum, its sum and the scale of its output are numbers of the lane, the probabilities are the next product's operand as
// they lie, and only the tile in LDS is read both along its rows and along its columns.
//
// A product of matrices multiplies every pair: 0 x infinity where a pair does not see each other.  Tiles that are partly hidden and hold
// something that is not finite are therefore multiplied without that, which is added afterwards (leave_finite, add_not_finite), so that NaN and
// infinities reach only the tokens that see them.
#ifndef SIG_WINDOW_H
#define SIG_WINDOW_H

#include <cfloat>

#include "sig_internal.h"
#include "sig_tiles.h"

namespace sig {

constexpr int kWindowThreads = 256, kWindowWaves = kWindowThreads / 64;

struct WindowArgs {
    const void *q, *k, *v;                // [B][T][heads or heads / group][.]
    int64_t qs[3], ks[3], vs[3];          // strides in values: batch, token, head
    void *out;                            // [B][T][heads][V], contiguous
    float2 *stats;                        // [B][heads][T]: m in powers of two, r; may be null in the forward pass
    const int64_t *lengths;               // [B], or null: T
    // of the gradient
    const void *grad_out;                 // as `out`
    void *grad_q, *grad_k, *grad_v;       // as q, k, v, contiguous
    float *delta;                         // [B][heads][T]: D
    int64_t B;
    int T, heads, group, K, V;
    int window, sinks;                    // at most T
    float scale, power;                   // c; |c| log2(e)
    int negated;                          // c < 0: the wavefront's own keys or queries change sign instead
    int tiles;                            // workgroups of a head
};

// What a workgroup works on, and the tiles of `N` tokens that its first to last token (lo ... hi - 1) have to do with
struct WindowPlace {
    int64_t b;
    int head, tile, n;      // n: tokens of the sequence
};

// Workgroups that follow one another take the last tiles of all heads first, which have the most to do where everything is seen.
// Eight dies take workgroups in turn, each with a cache of its own: where heads are a multiple of eight, a head's workgroups stay on one.
__device__ inline bool window_place(const WindowArgs &A, int heads, WindowPlace &p)
{
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, lines = A.B * heads;
    if (id >= lines * A.tiles) return false;
    int64_t line, tile;
    if (lines % 8 == 0) {
        const int64_t turn = id / 8;
        tile = turn % A.tiles;
        line = turn / A.tiles * 8 + id % 8;
    } else {
        tile = id / lines;
        line = id % lines;
    }
    p.tile = A.tiles - 1 - (int)tile;
    p.b = line / heads;
    p.head = (int)(line % heads);
    const int64_t n = A.lengths ? A.lengths[p.b] : A.T;
    p.n = n < 0 ? 0 : n > A.T ? A.T : (int)n;
    return true;
}

// Tiles of N keys that queries lo ... hi - 1 see: number j of `count` begins at key at(j)
template <int N>
struct KeyTiles {
    int front, first, count;      // the first tokens' tiles, then those from number `first` on
    __device__ KeyTiles(const WindowArgs &A, int lo, int hi)
    {
        const int low = max(0, lo + 1 - A.window);
        front = (min(A.sinks, low) + N - 1) / N;
        first = max(low / N, front);
        count = front + (hi + N - 1) / N - first;
    }
    __device__ int at(int j) const { return (j < front ? j : first + j - front) * N; }
};

struct Seen {
    int window, sinks;
    // (all of it compared: branches for single pairs cost more than the comparisons)
    __device__ bool operator()(int query, int key) const { return (key <= query) & ((query - key < window) | (key < sinks)); }
    // of queries q0 ... q1 and keys k0 ... k1
    __device__ bool all(int q0, int q1, int k0, int k1) const { return k1 <= q0 && (q1 - k0 < window || k1 < sinks); }
    __device__ bool none(int q0, int q1, int k0, int k1) const { return k0 > q1 || (k1 <= q0 - window && k0 >= sinks); }
};

// The wavefront's results, line l % M of a lane: acc[t] holds components t M + row_of(lane, i)
template <typename X, int D, typename T>
__device__ inline void store_line(T *line, int dim, int lane, const typename X::Result *acc, float scale)
{
#pragma unroll
    for (int t = 0; t < D / X::M; ++t)
#pragma unroll
        for (int i = 0; i < X::REGS; i += 4) {
            const int c = t * X::M + X::row_of(lane, i);
            Pack<T, 4> four;
#pragma unroll
            for (int j = 0; j < 4; ++j) four.v[j] = from_float<T>(acc[t][i + j] * scale);
            if (c + 4 <= dim) {
                store_pack(line + c, four);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < dim) line[c + j] = four.v[j];
            }
        }
}

template <typename T>
__device__ inline void zero_rows(T *first, int64_t stride, int dim, int from, int to)
{
    for (int64_t i = threadIdx.x; i < (int64_t)(to - from) * dim; i += kWindowThreads) first[(from + i / dim) * stride + i % dim] = from_float<T>(0.0f);
}

// ---------------------------------------------------------------- forward
template <typename T, typename X, int D, int N>
__global__ __launch_bounds__(kWindowThreads, D * sizeof(typename X::E) <= 256 ? 2 : 1) void sig_window_forward_kernel(WindowArgs A)
{
    using E = typename X::E;
    constexpr int M = X::M, ROWS = kWindowWaves * M, KEYS = N / M, STEPS = D / X::STEP, OUT = D / M;
    __shared__ __attribute__((aligned(16))) E keys[N * LdsTile<E, D>::PITCH];
    __shared__ __attribute__((aligned(16))) E values[N * LdsTile<E, D>::PITCH];
    __shared__ int spoilt[2];
    WindowPlace p;
    if (!window_place(A, A.heads, p)) return;
    const int lane = threadIdx.x % 64, lo = p.tile * ROWS, end = min(lo + ROWS, A.T);
    T *out = (T *)A.out + ((p.b * A.T) * A.heads + p.head) * A.V;
    const int64_t out_stride = (int64_t)A.heads * A.V;
    if (lo >= p.n) {
        zero_rows(out, out_stride, A.V, lo, end);
        return;
    }
    const int hi = min(end, p.n), shared = p.head / A.group;
    const T *k = (const T *)A.k + p.b * A.ks[0] + shared * A.ks[2], *v = (const T *)A.v + p.b * A.vs[0] + shared * A.vs[2];
    const int own = lo + threadIdx.x / 64 * M, line = own + lane % M;
    const bool there = line < p.n;
    typename X::Frag q[STEPS];
    fragments_of<X, STEPS>(q, lane, (const T *)A.q + p.b * A.qs[0] + (there ? line : lo) * A.qs[1] + p.head * A.qs[2], A.K, there, A.negated);
    const Seen seen = {A.window, A.sinks};
    const KeyTiles<N> tiles(A, lo, hi);
    TileMover<T, E, D, N, kWindowThreads> key_tile, value_tile;
    auto load = [&](int j) {
        const int at = tiles.at(j);
        key_tile.load(k + at * A.ks[1], A.ks[1], A.K, p.n - at);
        value_tile.load(v + at * A.vs[1], A.vs[1], A.V, p.n - at);
    };
    typename X::Result acc[OUT] = {};
    float m = -INFINITY, sum = 0.0f;      // of the lane's own part of its line
    if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
    load(0);
    for (int j = 0; j < tiles.count; ++j) {
        const int at = tiles.at(j);
        __syncthreads();
        key_tile.store(keys, A.K, p.n - at);
        value_tile.store(values, A.V, p.n - at);
        // (a tile that is partly hidden from some wavefront)
        if (!seen.all(lo, hi - 1, at, at + N - 1) && value_tile.spoilt(A.V, p.n - at)) spoilt[j & 1] = 1;
        if (threadIdx.x == 0) spoilt[~j & 1] = 0;
        __syncthreads();
        if (j + 1 < tiles.count) load(j + 1);
        const bool whole = seen.all(own, own + M - 1, at, at + N - 1), careful = spoilt[j & 1];
        const bool none = seen.none(own, min(own + M, hi) - 1, at, at + N - 1);
        typename X::Frag probabilities[N / X::STEP];
        if (!none) {
        typename X::Result s[KEYS] = {};
        product_of_rows<X, D, KEYS>(lane, keys, q, s);
        float most = -INFINITY;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                const bool ok = whole | seen(line, at + t * M + X::row_of(lane, i));
                s[t][i] = ok ? s[t][i] : -INFINITY;
                most = fmaxf(most, s[t][i]);
            }
        most = over_column<M>(most, fmaxf);
        const float next = fmaxf(m, most * A.power), base = next == -INFINITY ? 0.0f : next;      // (nothing seen so far: all p are 0)
        const float shrink = __builtin_amdgcn_exp2f(m - base);
        m = next;
        float part = 0.0f;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], A.power, -base));
                part += s[t][i];
            }
        sum = fmaf(sum, shrink, part);
#pragma unroll
        for (int t = 0; t < OUT; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) acc[t][i] *= shrink;
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) probabilities[step] = X::of_results(s, step);
        }
        if (careful) leave_finite<E, D, N, kWindowThreads>(values);
        if (!none) product_along_rows<X, D, N / X::STEP>(lane, values, probabilities, acc);
        if (careful) add_not_finite<X, D, N, kWindowThreads, false>(lane, values, v + at * A.vs[1], A.vs[1], A.V, p.n - at, none, acc, [&](int r) { return seen(line, at + r); });
    }
    sum = over_column<M>(sum, [](float a, float b) { return a + b; });
    const float r = 1.0f / sum;
    if (there) {
        store_line<X, D>(out + line * out_stride, A.V, lane, acc, r);
        if (A.stats && lane < M) A.stats[(p.b * A.heads + p.head) * A.T + line] = make_float2(m == -INFINITY ? 0.0f : m, r);
    }
    if (hi < end) zero_rows(out, out_stride, A.V, hi, end);
}

// ---------------------------------------------------------------- gradient of the queries, and D
template <typename T, typename X, int D, int N>
__global__ __launch_bounds__(kWindowThreads, D * sizeof(typename X::E) <= 128 ? 2 : 1) void sig_window_query_gradient_kernel(WindowArgs A)
{
    using E = typename X::E;
    constexpr int M = X::M, ROWS = kWindowWaves * M, KEYS = N / M, STEPS = D / X::STEP, OUT = D / M;
    __shared__ __attribute__((aligned(16))) E keys[N * LdsTile<E, D>::PITCH];
    __shared__ __attribute__((aligned(16))) E values[N * LdsTile<E, D>::PITCH];
    __shared__ int spoilt[2];
    WindowPlace p;
    if (!window_place(A, A.heads, p)) return;
    const int lane = threadIdx.x % 64, lo = p.tile * ROWS, end = min(lo + ROWS, A.T);
    T *out = (T *)A.grad_q + ((p.b * A.T) * A.heads + p.head) * A.K;
    const int64_t out_stride = (int64_t)A.heads * A.K;
    if (lo >= p.n) {
        zero_rows(out, out_stride, A.K, lo, end);
        return;
    }
    const int hi = min(end, p.n), shared = p.head / A.group;
    const T *k = (const T *)A.k + p.b * A.ks[0] + shared * A.ks[2], *v = (const T *)A.v + p.b * A.vs[0] + shared * A.vs[2];
    const int own = lo + threadIdx.x / 64 * M, line = own + lane % M;
    const bool there = line < p.n;
    typename X::Frag q[STEPS], g[STEPS];
    fragments_of<X, STEPS>(q, lane, (const T *)A.q + p.b * A.qs[0] + (there ? line : lo) * A.qs[1] + p.head * A.qs[2], A.K, there, A.negated);
    const int64_t upstream = ((p.b * A.T + (there ? line : lo)) * A.heads + p.head) * A.V, place = (p.b * A.heads + p.head) * A.T + line;
    fragments_of<X, STEPS>(g, lane, (const T *)A.grad_out + upstream, A.V, there, false);
    float delta = 0.0f;
    {
        // (the output as the forward pass rounded it)
        typename X::Frag o[STEPS];
        fragments_of<X, STEPS>(o, lane, (const T *)A.out + upstream, A.V, there, false);
#pragma unroll
        for (int j = 0; j < STEPS; ++j)
#pragma unroll
            for (int e = 0; e < X::GROUP; ++e) delta = fmaf((float)o[j][e], (float)g[j][e], delta);
        delta = over_column<M>(delta, [](float a, float b) { return a + b; });
    }
    float2 stats = make_float2(0.0f, 0.0f);
    if (there) {
        stats = A.stats[place];
        if (lane < M) A.delta[place] = delta;
    }
    const Seen seen = {A.window, A.sinks};
    const KeyTiles<N> tiles(A, lo, hi);
    TileMover<T, E, D, N, kWindowThreads> key_tile, value_tile;
    auto load = [&](int j) {
        const int at = tiles.at(j);
        key_tile.load(k + at * A.ks[1], A.ks[1], A.K, p.n - at);
        value_tile.load(v + at * A.vs[1], A.vs[1], A.V, p.n - at);
    };
    typename X::Result acc[OUT] = {};
    if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
    load(0);
    for (int j = 0; j < tiles.count; ++j) {
        const int at = tiles.at(j);
        __syncthreads();
        key_tile.store(keys, A.K, p.n - at);
        value_tile.store(values, A.V, p.n - at);
        if (!seen.all(lo, hi - 1, at, at + N - 1) && key_tile.spoilt(A.K, p.n - at)) spoilt[j & 1] = 1;
        if (threadIdx.x == 0) spoilt[~j & 1] = 0;
        __syncthreads();
        if (j + 1 < tiles.count) load(j + 1);
        const bool whole = seen.all(own, own + M - 1, at, at + N - 1), careful = spoilt[j & 1];
        const bool none = seen.none(own, min(own + M, hi) - 1, at, at + N - 1);
        typename X::Frag terms[N / X::STEP];
        if (!none) {
        typename X::Result s[KEYS] = {}, u[KEYS] = {};
        product_of_rows<X, D, KEYS>(lane, keys, q, s);
        product_of_rows<X, D, KEYS>(lane, values, g, u);
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                const float probability = __builtin_amdgcn_exp2f(fmaf(s[t][i], A.power, -stats.x)) * stats.y;
                const bool ok = whole | seen(line, at + t * M + X::row_of(lane, i));
                u[t][i] = ok ? probability * (u[t][i] - delta) : 0.0f;
            }
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) terms[step] = X::of_results(u, step);
        }
        if (careful) leave_finite<E, D, N, kWindowThreads>(keys);
        if (!none) product_along_rows<X, D, N / X::STEP>(lane, keys, terms, acc);
        if (careful) add_not_finite<X, D, N, kWindowThreads, true>(lane, keys, k + at * A.ks[1], A.ks[1], A.K, p.n - at, none, acc, [&](int r) { return seen(line, at + r); });
    }
    if (there) store_line<X, D>(out + line * out_stride, A.K, lane, acc, A.scale);
    if (hi < end) zero_rows(out, out_stride, A.K, hi, end);
}

// ---------------------------------------------------------------- gradient of keys and values
// A wavefront's own lines are keys; queries and upstream gradients of all heads that share them come as tiles, one head after the other, so
// that the sum over these heads is one of registers.
template <typename T, typename X, int D, int N>
__global__ __launch_bounds__(kWindowThreads, 1) void sig_window_key_gradient_kernel(WindowArgs A)
{
    using E = typename X::E;
    constexpr int M = X::M, ROWS = kWindowWaves * M, QUERIES = N / M, STEPS = D / X::STEP, OUT = D / M;
    __shared__ __attribute__((aligned(16))) E queries[N * LdsTile<E, D>::PITCH];
    __shared__ __attribute__((aligned(16))) E upstream[N * LdsTile<E, D>::PITCH];
    __shared__ __attribute__((aligned(16))) float most[N], inverse[N], delta[N];
    __shared__ int spoilt[2];
    WindowPlace p;
    const int shared_heads = A.heads / A.group;
    if (!window_place(A, shared_heads, p)) return;
    const int lane = threadIdx.x % 64, lo = p.tile * ROWS, end = min(lo + ROWS, A.T);
    T *out_k = (T *)A.grad_k + ((p.b * A.T) * shared_heads + p.head) * A.K, *out_v = (T *)A.grad_v + ((p.b * A.T) * shared_heads + p.head) * A.V;
    const int64_t k_stride = (int64_t)shared_heads * A.K, v_stride = (int64_t)shared_heads * A.V, g_stride = (int64_t)A.heads * A.V;
    if (lo >= p.n) {
        zero_rows(out_k, k_stride, A.K, lo, end);
        zero_rows(out_v, v_stride, A.V, lo, end);
        return;
    }
    const int hi = min(end, p.n);
    const int own = lo + threadIdx.x / 64 * M, line = own + lane % M;
    const bool there = line < p.n;
    typename X::Frag k[STEPS], v[STEPS];
    fragments_of<X, STEPS>(k, lane, (const T *)A.k + p.b * A.ks[0] + (there ? line : lo) * A.ks[1] + p.head * A.ks[2], A.K, there, A.negated);
    fragments_of<X, STEPS>(v, lane, (const T *)A.v + p.b * A.vs[0] + (there ? line : lo) * A.vs[1] + p.head * A.vs[2], A.V, there, false);
    const Seen seen = {A.window, A.sinks};
    // queries from lo on; where no key is one of the first tokens, those that have the last one in their window
    const int first = lo / N, last = (lo < A.sinks ? p.n : (int)min((int64_t)p.n, (int64_t)hi - 1 + A.window)) - 1, tiles = last / N - first + 1, count = tiles * A.group;
    TileMover<T, E, D, N, kWindowThreads> query_tile, upstream_tile;
    float2 stats_tile;
    float delta_tile;
    auto load = [&](int j) {
        const int head = p.head * A.group + j / tiles, at = (first + j % tiles) * N;
        query_tile.load((const T *)A.q + p.b * A.qs[0] + head * A.qs[2] + at * A.qs[1], A.qs[1], A.K, p.n - at);
        upstream_tile.load((const T *)A.grad_out + ((p.b * A.T + at) * A.heads + head) * A.V, g_stride, A.V, p.n - at);
        stats_tile = make_float2(0.0f, 0.0f);
        delta_tile = 0.0f;
        if (threadIdx.x < N && at + (int)threadIdx.x < p.n) {
            const int64_t place = (p.b * A.heads + head) * A.T + at + threadIdx.x;
            stats_tile = A.stats[place];
            delta_tile = A.delta[place];
        }
    };
    typename X::Result acc_k[OUT] = {}, acc_v[OUT] = {};
    if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
    load(0);
    for (int j = 0; j < count; ++j) {
        const int at = (first + j % tiles) * N;
        __syncthreads();
        query_tile.store(queries, A.K, p.n - at);
        upstream_tile.store(upstream, A.V, p.n - at);
        if (threadIdx.x < N) {
            most[threadIdx.x] = stats_tile.x;
            inverse[threadIdx.x] = stats_tile.y;
            delta[threadIdx.x] = delta_tile;
        }
        if (!seen.all(at, at + N - 1, lo, lo + ROWS - 1) && (query_tile.spoilt(A.K, p.n - at) || upstream_tile.spoilt(A.V, p.n - at))) spoilt[j & 1] = 1;
        if (threadIdx.x == 0) spoilt[~j & 1] = 0;
        __syncthreads();
        if (j + 1 < count) load(j + 1);
        const bool whole = at + N <= p.n && seen.all(at, at + N - 1, own, own + M - 1);
        const bool none = seen.none(at, min(at + N, p.n) - 1, own, min(own + M, hi) - 1), careful = spoilt[j & 1];
        typename X::Frag weights[N / X::STEP], terms[N / X::STEP];
        if (!none) {
        typename X::Result s[QUERIES] = {}, u[QUERIES] = {};
        product_of_rows<X, D, QUERIES>(lane, queries, k, s);
        product_of_rows<X, D, QUERIES>(lane, upstream, v, u);
#pragma unroll
        for (int t = 0; t < QUERIES; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                const int row = t * M + X::row_of(lane, i);
                const bool ok = whole | ((at + row < p.n) & seen(at + row, line));
                s[t][i] = ok ? __builtin_amdgcn_exp2f(fmaf(s[t][i], A.power, -most[row])) * inverse[row] : 0.0f;
                u[t][i] = ok ? s[t][i] * (u[t][i] - delta[row]) : 0.0f;
            }
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) {
            weights[step] = X::of_results(s, step);
            terms[step] = X::of_results(u, step);
        }
        }
        if (careful) {
            leave_finite<E, D, N, kWindowThreads>(queries);
            leave_finite<E, D, N, kWindowThreads>(upstream);
        }
        if (!none) {
            product_along_rows<X, D, N / X::STEP>(lane, upstream, weights, acc_v);
            product_along_rows<X, D, N / X::STEP>(lane, queries, terms, acc_k);
        }
        if (careful) {
            const int head = p.head * A.group + j / tiles, n = p.n - at;
            auto sees = [&](int r) { return seen(at + r, line); };
            add_not_finite<X, D, N, kWindowThreads, false>(lane, upstream, (const T *)A.grad_out + ((p.b * A.T + at) * A.heads + head) * A.V, g_stride, A.V, n, none, acc_v, sees);
            add_not_finite<X, D, N, kWindowThreads, true>(lane, queries, (const T *)A.q + p.b * A.qs[0] + head * A.qs[2] + at * A.qs[1], A.qs[1], A.K, n, none, acc_k, sees);
        }
    }
    if (there) {
        store_line<X, D>(out_k + line * k_stride, A.K, lane, acc_k, A.scale);
        store_line<X, D>(out_v + line * v_stride, A.V, lane, acc_v, 1.0f);
    }
    if (hi < end) {
        zero_rows(out_k, k_stride, A.K, hi, end);
        zero_rows(out_v, v_stride, A.V, hi, end);
    }
}

// ---------------------------------------------------------------- launches
enum WindowPass { WINDOW_FORWARD, WINDOW_QUERY_GRADIENT, WINDOW_KEY_GRADIENT };

hipError_t launch_window_f32(const WindowArgs &A, WindowPass pass, hipStream_t st);
hipError_t launch_window_bf16(const WindowArgs &A, WindowPass pass, hipStream_t st);
hipError_t launch_window_f16(const WindowArgs &A, WindowPass pass, hipStream_t st);

// T: in memory; E: of the products
template <typename T, typename E>
hipError_t launch_window(WindowArgs A, WindowPass pass, hipStream_t st)
{
    const int dim = A.K > A.V ? A.K : A.V;
    auto go = [&](auto x, auto d) {
        using X = typename decltype(x)::type;
        constexpr int D = decltype(d)::value, ROWS = kWindowWaves * X::M, BYTES = D * (int)sizeof(E);
        // tokens of a tile
        constexpr int N = BYTES > 512 ? 16 : BYTES > 128 ? 32 : 64, GRADIENT = BYTES > 512 ? 16 : 32;
        A.tiles = (A.T + ROWS - 1) / ROWS;
        const int64_t blocks = A.B * (pass == WINDOW_KEY_GRADIENT ? A.heads / A.group : A.heads) * A.tiles;
        const int64_t across = ((int64_t)1 << 32) / kWindowThreads - 1;      // (a launch holds fewer than 2^32 threads along an axis)
        const dim3 grid((unsigned)(blocks < across ? blocks : across), (unsigned)((blocks + across - 1) / across));
        if (pass == WINDOW_FORWARD) sig_window_forward_kernel<T, X, D, N><<<grid, kWindowThreads, 0, st>>>(A);
        else if (pass == WINDOW_QUERY_GRADIENT) sig_window_query_gradient_kernel<T, X, D, N><<<grid, kWindowThreads, 0, st>>>(A);
        else sig_window_key_gradient_kernel<T, X, D, GRADIENT><<<grid, kWindowThreads, 0, st>>>(A);
    };
    if (dim <= 64) go(Tag<Tiles<E>>(), std::integral_constant<int, 64>());
    else if (dim <= 128) go(Tag<Tiles<E>>(), std::integral_constant<int, 128>());
    else go(Tag<SmallTiles<E>>(), std::integral_constant<int, 256>());
    return hipGetLastError();
}

}  // namespace sig
#endif
