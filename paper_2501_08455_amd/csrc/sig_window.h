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

// What the rounding of an output to 16 bits leaves, in 8 bits (5 of exponent), times 2^14.  D = g . o decides the gradient where a token sees few others,
// so that there the output's rounding would cost as much as all others together: window 4, 128 components, the gradient of queries is off by 1.75 of what its own
// rounding comes to without the rest, and by 1.43 with it.  Three digits of it are enough.  Outputs of 2^-16 to 2^10 have them, beyond it only helps less.
using Rest = uint8_t;
constexpr float kRestScale = 16384.0f, kMostRest = 57344.0f;

__device__ inline unsigned rest_of(float low, float high, unsigned other, bool upper)
{
    low = __builtin_amdgcn_fmed3f(low * kRestScale, -kMostRest, kMostRest);
    high = __builtin_amdgcn_fmed3f(high * kRestScale, -kMostRest, kMostRest);
    return upper ? __builtin_amdgcn_cvt_pk_bf8_f32(low, high, other, true) : __builtin_amdgcn_cvt_pk_bf8_f32(low, high, other, false);
}
template <int BYTE>
__device__ inline float rest_value(unsigned four)
{
    return __builtin_amdgcn_cvt_f32_bf8(four, BYTE) * (1.0f / kRestScale);
}

struct WindowArgs {
    const void *q, *k, *v;                // [B][T][heads or heads / group][.]
    int64_t qs[3], ks[3], vs[3];          // strides in values: batch, token, head
    void *out;                            // [B][T][heads][V], contiguous
    float2 *stats;                        // [B][heads][T]: m in powers of two, r; may be null in the forward pass
    Rest *rest;                           // as `out`, of 16 bits: what its rounding left; null where stats is
    const int64_t *lengths;               // [B], or null: T
    // of the gradient
    const void *grad_out;                 // as `out`
    void *grad_q, *grad_k, *grad_v;       // as q, k, v, contiguous
    float *delta;                         // [B][heads][T]: D
    // Keys' gradients that are cut along the queries: `cut` tiles into `parts` each, whose sums for the first `joined` keys are added up from scratch,
    // [B][shared heads][cut][parts][rows of a tile][K + V].  Either all tiles, evenly, where there are few, or those of the first tokens, which every query sees
    float *sums;
    int cut, parts, joined, even;
    // Queries that are few are cut along their keys: `splits` pieces of each tile's keys, [B][heads][splits][T] lines of what each adds up to: V values of the output, not yet
    // divided, with the maximum and the sum that belong to them, or K of the queries' gradient
    float *pieces;
    int splits;
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
    int split;              // which piece of the keys
};

// Workgroups that follow one another take the last tiles first, which have the most to do where everything is seen.
// Eight dies take workgroups in turn, each with a cache of its own: where heads are a multiple of eight, a head's workgroups stay on one.
__device__ inline bool window_place(const WindowArgs &A, int heads, WindowPlace &p)
{
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, lines = A.B * heads;
    const int64_t pieces = (int64_t)A.tiles * A.splits;
    if (id >= lines * pieces) return false;
    int64_t line, piece;
    if (lines % 8 == 0) {
        const int64_t turn = id / 8;
        piece = turn % pieces;
        line = turn / pieces * 8 + id % 8;
    } else {
        piece = id / lines;
        line = id % lines;
    }
    p.tile = A.tiles - 1 - (int)(piece / A.splits);
    p.split = (int)(piece % A.splits);
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
    // the first tile of piece number i
    __device__ int piece(int i, int splits) const { return (int)((int64_t)count * i / splits); }
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

// ... and what its rounding to T leaves
template <typename X, int D, typename T>
__device__ inline void store_rest(Rest *line, int dim, int lane, const typename X::Result *acc, float scale)
{
#pragma unroll
    for (int t = 0; t < D / X::M; ++t)
#pragma unroll
        for (int i = 0; i < X::REGS; i += 4) {
            const int c = t * X::M + X::row_of(lane, i);
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = acc[t][i + j] * scale;
                x[j] -= to_float(from_float<T>(x[j]));
            }
            const unsigned four = rest_of(x[2], x[3], rest_of(x[0], x[1], 0, false), true);
            if (c + 4 <= dim) {
                store_pack(line + c, __builtin_bit_cast(Pack<Rest, 4>, four));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < dim) line[c + j] = (Rest)(four >> (8 * j));
            }
        }
}

template <int THREADS = kWindowThreads, typename T>
__device__ inline void zero_rows(T *first, int64_t stride, int dim, int from, int to)
{
    for (int64_t i = threadIdx.x; i < (int64_t)(to - from) * dim; i += THREADS) first[(from + i / dim) * stride + i % dim] = from_float<T>(0.0f);
}

// The maximum that everything is scaled with may stay behind by a power of two, so that what is added up so far need not be touched each time it grows.  Float16's probabilities
// are lifted (lifted_base), to 2^15 at most with a maximum that stays behind: those down to e^-19 of the largest are no subnormal numbers.  (By 2^7, with a maximum that stays
// behind by 2^8: one score 18 above 699 others whose values are all that counts, the output 6.8e-3 off instead of 2.9e-4, its own rounding; 20 above 5.0e-2 instead of 4.9e-4.  8 x 4,096
// tokens, 16 heads of 128, window 1,024: 448 instead of 458 us.)
template <typename E>
constexpr float kBehind = std::is_same_v<E, f16> ? 1.0f : 8.0f;
constexpr int kLift = 14;
constexpr int kFewTokens = 16;

// Gradient terms in float16 have no scale that suits all of them: each lane (a line of the result) has a power of two of its own, `factor`, which
// keeps its largest term so far within 2^15 and above 2^-7 of that when it is chosen.  Returns what the sums so far are to be multiplied with.
struct TermScale {
    float factor = 0.0f;      // none yet

    template <int M, int COUNT, typename Result>
    __device__ bool grown(const Result *u, float *shrink)
    {
        float most = 0.0f;
#pragma unroll
        for (int t = 0; t < COUNT; ++t)
#pragma unroll
            for (int i = 0; i < (int)(sizeof(Result) / 4); ++i) most = fmaxf(most, fabsf(u[t][i]));
        most = over_column<M>(most, fmaxf);
        const bool change = (most > 0.0f) & (most < INFINITY) & ((factor == 0.0f) | (most * factor > 32768.0f));
        *shrink = 1.0f;
        if (!__any(change)) return false;
        if (change) {
            int exponent = (int)(__builtin_bit_cast(unsigned, most) >> 23) - 127;
            exponent = min(max(8 - exponent, -120), 120);
            const float next = __builtin_bit_cast(float, (unsigned)(exponent + 127) << 23);
            *shrink = factor == 0.0f ? 1.0f : next / factor;
            factor = next;
        }
        return true;
    }
    __device__ float back() const { return factor == 0.0f ? 1.0f : 1.0f / factor; }
};

// ---------------------------------------------------------------- forward
template <typename T, typename X, int D, int N, bool WHOLE>
__global__ __launch_bounds__(kWindowThreads, D * X::PLANES * sizeof(typename X::E) <= 512 ? 2 : 1) void sig_window_forward_kernel(WindowArgs A)
{
    using E = typename X::E;
    constexpr int M = X::M, ROWS = kWindowWaves * M, KEYS = N / M, STEPS = D / X::STEP, OUT = D / M, SIZE = N * X::template Tile<D>::PITCH;
    __shared__ __attribute__((aligned(16))) E keys[2 * SIZE];
    __shared__ __attribute__((aligned(16))) E values[2 * SIZE];
    __shared__ int spoilt[2];      // 1 + the number of a tile that is partly hidden and holds something that is not finite
    WindowPlace p;
    if (!window_place(A, A.heads, p)) return;
    const int lane = threadIdx.x % 64, lo = p.tile * ROWS, end = min(lo + ROWS, A.T);
    T *out = (T *)A.out + ((p.b * A.T) * A.heads + p.head) * A.V;
    const int64_t out_stride = (int64_t)A.heads * A.V;
    if (lo >= p.n) {
        if (p.split == 0) zero_rows(out, out_stride, A.V, lo, end);
        return;
    }
    const int hi = min(end, p.n), shared = p.head / A.group;
    const T *k = (const T *)A.k + p.b * A.ks[0] + shared * A.ks[2], *v = (const T *)A.v + p.b * A.vs[0] + shared * A.vs[2];
    const int own = lo + (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64) * M, line = own + lane % M;
    const bool there = line < p.n;
    typename X::Frag q[STEPS];
    fragments_of<X, STEPS>(q, lane, (const T *)A.q + p.b * A.qs[0] + (there ? line : lo) * A.qs[1] + p.head * A.qs[2], A.K, there, A.negated);
    const Seen seen = {A.window, A.sinks};
    const KeyTiles<N> tiles(A, lo, hi);
    const int begin = tiles.piece(p.split, A.splits), until = tiles.piece(p.split + 1, A.splits);
    TileMover<T, X, D, N, kWindowThreads, WHOLE> key_tile, value_tile;
    auto load = [&](int j) {
        const int at = tiles.at(j);
        key_tile.load(k + at * A.ks[1], A.ks[1], A.K, p.n - at);
        value_tile.load(v + at * A.vs[1], A.vs[1], A.V, p.n - at);
    };
    auto store = [&](int j, auto careful) {
        constexpr bool NANS = decltype(careful)::value;
        const int at = tiles.at(j);
        key_tile.template store<NANS>(keys + (j & 1) * SIZE, A.K, p.n - at);
        value_tile.store(values + (j & 1) * SIZE, A.V, p.n - at);
        // (float32's parts: infinities that all see as well, which are no products of theirs)
        if constexpr (X::PLANES > 1) {
            if (key_tile.spoilt(A.K, p.n - at) || value_tile.spoilt(A.V, p.n - at)) spoilt[j & 1] = j + 1;
        } else {
            if (!seen.all(lo, hi - 1, at, at + N - 1) && value_tile.spoilt(A.V, p.n - at)) spoilt[j & 1] = j + 1;
        }
    };
    typename X::Result acc[OUT] = {};
    float m = -INFINITY, sum = 0.0f;      // the base that its line is scaled with; of the lane's own part of it
    typename X::Frag probabilities[N / X::STEP];
    // the probabilities of tile j, and the running maximum and sum
    auto weigh = [&](int at, const E *keys, auto careful) {
        typename X::Result s[KEYS] = {};
        product_of_rows<X, D, KEYS, WHOLE>(lane, keys, q, s, A.K);
        if constexpr (decltype(careful)::value) settle_infinities<X, D, KEYS>(lane, keys, q, s);
        if (!seen.all(own, own + M - 1, at, at + N - 1)) {
#pragma unroll
            for (int t = 0; t < KEYS; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) s[t][i] = seen(line, at + t * M + X::row_of(lane, i)) ? s[t][i] : -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) most = fmaxf(most, s[t][i]);
        most = over_column<M>(most, fmaxf);
        const float next = fmaxf(m, lifted_base<E, kLift>(most * A.power));
        if (__any(next > m + kBehind<E>)) {
            const float shrink = __builtin_amdgcn_exp2f(m - (next == -INFINITY ? 0.0f : next));
            m = next;
            sum *= shrink;
#pragma unroll
            for (int t = 0; t < OUT; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) acc[t][i] *= shrink;
        }
        const float base = m == -INFINITY ? 0.0f : m;      // (nothing seen so far: all p are 0)
        float part = 0.0f;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], A.power, -base));
                part += s[t][i];
            }
        sum += part;
        // 16 bits: rounded to the operands' type for their product, while the sum that divides them stays float32's.  Outputs then are 2.4e-3 off in bfloat16, of which their own rounding is
        // 1.7e-3 (window 1,024 and 4,096).  A second part of each, as attention over a cache has it, leaves just that, but is a product more beside two: 65,536 tokens, 16 heads (4 shared) of
        // 128, window 4,096 2,670 -> 3,520 us, 8 x 4,096, 16 heads, window 1,024 482 -> 598.
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) probabilities[step] = X::of_results(s, step);
    };
    auto none = [&](int at) { return own >= hi || seen.none(own, min(own + M, hi) - 1, at, at + N - 1); };
    // Tile j is in LDS, tile j + 1 on its way to registers: it goes to LDS's other half in the middle of tile j's work.  Spoilt tiles are left out, and
    // taken by themselves afterwards (a branch in the middle would cost every tile its registers)
    bool left_out = false;
    if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
    if (begin < until) load(begin);
    __syncthreads();
    if (begin < until) store(begin, std::false_type());
    if (begin + 1 < until) load(begin + 1);
    for (int j = begin; j < until; ++j) {
        const int at = tiles.at(j), half = (j & 1) * SIZE;
        __syncthreads();
        const bool bad = __builtin_amdgcn_readfirstlane(spoilt[j & 1]) == j + 1, skip = bad || none(at);
        left_out |= bad;
        if (!skip) weigh(at, keys + half, std::false_type());
        if (j + 1 < until) store(j + 1, std::false_type());
        if (j + 2 < until) load(j + 2);
        if (!skip) product_along_rows<X, D, N / X::STEP, WHOLE>(lane, values + half, probabilities, acc, A.V);
    }
    if (left_out) {
#pragma unroll 1
        for (int j = begin; j < until; ++j) {
            const int at = tiles.at(j);
            E *tile = values + (j & 1) * SIZE;
            __syncthreads();
            load(j);
            store(j, std::true_type());
            __syncthreads();
            if (spoilt[j & 1] != j + 1) continue;
            const bool skip = none(at);
            if (!skip) weigh(at, keys + (j & 1) * SIZE, std::true_type());
            leave_finite<X, D, N, kWindowThreads>(tile);
            if (!skip) product_along_rows<X, D, N / X::STEP, WHOLE>(lane, tile, probabilities, acc, A.V);
            add_not_finite<X, D, N, kWindowThreads, false>(lane, tile, v + at * A.vs[1], A.vs[1], A.V, p.n - at, skip, acc, [&](int r) { return seen(line, at + r); });
        }
    }
    sum = over_column<M>(sum, [](float a, float b) { return a + b; });
    if (A.splits > 1) {
        if (there) {
            float *piece = A.pieces + (((p.b * A.heads + p.head) * A.splits + p.split) * A.T + line) * (A.V + 2);
            store_line<X, D>(piece, A.V, lane, acc, 1.0f);
            if (lane < M) {
                piece[A.V] = m;
                piece[A.V + 1] = sum;
            }
        }
        if (hi < end && p.split == 0) zero_rows(out, out_stride, A.V, hi, end);
        return;
    }
    const float r = 1.0f / sum;
    if (there) {
        store_line<X, D>(out + line * out_stride, A.V, lane, acc, r);
        if constexpr (sizeof(T) == 2) {
            if (A.rest) store_rest<X, D, T>(A.rest + ((p.b * A.T + line) * A.heads + p.head) * A.V, A.V, lane, acc, r);
        }
        if (A.stats && lane < M) A.stats[(p.b * A.heads + p.head) * A.T + line] = make_float2(m == -INFINITY ? 0.0f : m, r);
    }
    if (hi < end) zero_rows(out, out_stride, A.V, hi, end);
}

// ---------------------------------------------------------------- gradient of the queries, and D
// Two workgroups a unit, where their registers fit (one, with the forward pass alike: 4 x 2,048 tokens, 16 heads (4 shared) of 256 bfloat16 495 instead of 310 us, with the gradient 1,621
// instead of 1,245; of 80 823 instead of 699; 199 x 6 tokens, 44 heads (11 shared) of 256 x 130 305 instead of 155)
template <typename X, int D, bool WHOLE>
constexpr bool kQueryPairs = X::PLANES > 1 ? D <= 64 : sizeof(typename X::E) == 2 && (WHOLE || X::M == 16 || D <= 96);

template <typename T, typename X, int D, int N, bool WHOLE>
__global__ __launch_bounds__(kWindowThreads, (kQueryPairs<X, D, WHOLE>) ? 2 : 1) void sig_window_query_gradient_kernel(WindowArgs A)
{
    using E = typename X::E;
    constexpr int M = X::M, ROWS = kWindowWaves * M, KEYS = N / M, STEPS = D / X::STEP, OUT = D / M, SIZE = N * X::template Tile<D>::PITCH;
    __shared__ __attribute__((aligned(16))) E keys[2 * SIZE];
    __shared__ __attribute__((aligned(16))) E values[2 * SIZE];
    __shared__ int spoilt[2];
    WindowPlace p;
    if (!window_place(A, A.heads, p)) return;
    const int lane = threadIdx.x % 64, lo = p.tile * ROWS, end = min(lo + ROWS, A.T);
    T *out = (T *)A.grad_q + ((p.b * A.T) * A.heads + p.head) * A.K;
    const int64_t out_stride = (int64_t)A.heads * A.K;
    if (lo >= p.n) {
        if (p.split == 0) zero_rows(out, out_stride, A.K, lo, end);
        return;
    }
    const int hi = min(end, p.n), shared = p.head / A.group;
    const T *k = (const T *)A.k + p.b * A.ks[0] + shared * A.ks[2], *v = (const T *)A.v + p.b * A.vs[0] + shared * A.vs[2];
    const int own = lo + (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64) * M, line = own + lane % M;
    const bool there = line < p.n;
    typename X::Frag q[STEPS], g[STEPS];
    fragments_of<X, STEPS>(q, lane, (const T *)A.q + p.b * A.qs[0] + (there ? line : lo) * A.qs[1] + p.head * A.qs[2], A.K, there, A.negated);
    const int64_t upstream = ((p.b * A.T + (there ? line : lo)) * A.heads + p.head) * A.V, place = (p.b * A.heads + p.head) * A.T + line;
    fragments_of<X, STEPS>(g, lane, (const T *)A.grad_out + upstream, A.V, there, false);
    float delta = 0.0f;
    {
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            typename X::Frag o;
            fragment_of<X>(&o, lane, j, (const T *)A.out + upstream, A.V, there);
            if constexpr (sizeof(T) == 2) {
                const int at = j * X::STEP + X::first_of(lane);
                uint64_t eight = 0;
                if (there && at + 8 <= A.V) {
                    eight = __builtin_bit_cast(uint64_t, load_pack<Rest, 8>(A.rest + upstream + at));
                } else if (there) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (at + e < A.V) eight |= (uint64_t)A.rest[upstream + at + e] << (8 * e);
                }
                const unsigned words[] = {(unsigned)eight, (unsigned)(eight >> 32)};
                float rest = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    rest = fmaf(rest_value<0>(words[h]), (float)g[j][4 * h], rest);
                    rest = fmaf(rest_value<1>(words[h]), (float)g[j][4 * h + 1], rest);
                    rest = fmaf(rest_value<2>(words[h]), (float)g[j][4 * h + 2], rest);
                    rest = fmaf(rest_value<3>(words[h]), (float)g[j][4 * h + 3], rest);
                }
                delta += rest;
            }
#pragma unroll
            for (int e = 0; e < X::GROUP; ++e) delta = fmaf(fragment_value(o, e), fragment_value(g[j], e), delta);
        }
        delta = over_column<M>(delta, [](float a, float b) { return a + b; });
    }
    float2 stats = make_float2(0.0f, 0.0f);
    if (there) stats = A.stats[place];
    const Seen seen = {A.window, A.sinks};
    const KeyTiles<N> tiles(A, lo, hi);
    const int begin = tiles.piece(p.split, A.splits), until = tiles.piece(p.split + 1, A.splits);
    TileMover<T, X, D, N, kWindowThreads, WHOLE, (X::PLANES > 1 && !WHOLE)> key_tile, value_tile;
    auto load = [&](int j) {
        const int at = tiles.at(j);
        key_tile.load(k + at * A.ks[1], A.ks[1], A.K, p.n - at);
        value_tile.load(v + at * A.vs[1], A.vs[1], A.V, p.n - at);
    };
    auto store = [&](int j, auto careful) {
        constexpr bool NANS = decltype(careful)::value;
        const int at = tiles.at(j);
        key_tile.template store<NANS>(keys + (j & 1) * SIZE, A.K, p.n - at);
        value_tile.store(values + (j & 1) * SIZE, A.V, p.n - at);
        if ((X::PLANES > 1 || !seen.all(lo, hi - 1, at, at + N - 1)) && key_tile.spoilt(A.K, p.n - at)) spoilt[j & 1] = j + 1;
    };
    auto none = [&](int at) { return own >= hi || seen.none(own, min(own + M, hi) - 1, at, at + N - 1); };
    // p (g . v - D) of a tile
    auto find_terms = [&](int at, const E *keys, const E *values, typename X::Result *u, auto careful) {
        typename X::Result s[KEYS] = {};
        product_of_rows<X, D, KEYS, WHOLE>(lane, keys, q, s, A.K);
        if constexpr (decltype(careful)::value) settle_infinities<X, D, KEYS>(lane, keys, q, s);
        product_of_rows<X, D, KEYS, WHOLE>(lane, values, g, u, A.V);
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) u[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], A.power, -stats.x)) * stats.y * (u[t][i] - delta);
        if (!seen.all(own, own + M - 1, at, at + N - 1)) {
#pragma unroll
            for (int t = 0; t < KEYS; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) u[t][i] = seen(line, at + t * M + X::row_of(lane, i)) ? u[t][i] : 0.0f;
        }
    };
    if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
    // Where no query of the workgroup sees more than a few tokens, D is also off by what the rounded probabilities made of the output, by as much as its own rounding would be.  (The first
    // few tokens of a longer sequence with a larger window see as few, but share their workgroup with others that see more, and go without.)
    // The terms' sum, which should be 0, is that error, so it is found first (window 3 of 24 components, bfloat16: gradients of queries and keys 1.50 of their
    // rounding off without it, 1.42 with it; it costs two of the three products once more, where there are few of them: 16 x 2,048 tokens, 16 heads of 64, both
    // passes 543 us with a window of 8, 493 without this with one of 17)
    if (sizeof(T) == 2 && min((int64_t)hi, (int64_t)A.window + A.sinks) <= kFewTokens) {
        float off = 0.0f;
#pragma unroll 1
        for (int j = 0; j < tiles.count; ++j) {
            if (!WHOLE) asm volatile("" : "+s"(A.K), "+s"(A.V));      // (else what depends on them is kept over the loop, in more registers than there are)
            __syncthreads();
            load(j);
            store(j, std::false_type());
            __syncthreads();
            if (none(tiles.at(j))) continue;
            typename X::Result u[KEYS] = {};
            find_terms(tiles.at(j), keys + (j & 1) * SIZE, values + (j & 1) * SIZE, u, std::false_type());
#pragma unroll
            for (int t = 0; t < KEYS; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) off += u[t][i];
        }
        delta += over_column<M>(off, [](float a, float b) { return a + b; });
        __syncthreads();
        if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
    }
    if (there && lane < M && p.split == 0) A.delta[place] = delta;
    typename X::Result acc[OUT] = {};
    TermScale scale;
    typename X::Frag terms[N / X::STEP];
    auto weigh = [&](int at, const E *keys, const E *values, auto careful) {
        typename X::Result u[KEYS] = {};
        find_terms(at, keys, values, u, careful);
        if constexpr (std::is_same_v<E, f16>) {
            float shrink;
            if (scale.grown<M, KEYS>(u, &shrink)) {
#pragma unroll
                for (int t = 0; t < OUT; ++t)
#pragma unroll
                    for (int i = 0; i < X::REGS; ++i) acc[t][i] *= shrink;
            }
#pragma unroll
            for (int t = 0; t < KEYS; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) u[t][i] *= scale.factor;
        }
        // (16 bits: rounded to the operands' type, as the forward pass's probabilities are, and for the same reason: a second part would be a product more beside three)
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) terms[step] = X::of_results(u, step);
    };
    bool left_out = false;
    if (begin < until) load(begin);
    __syncthreads();
    if (begin < until) store(begin, std::false_type());
    if (begin + 1 < until) load(begin + 1);
    for (int j = begin; j < until; ++j) {
        const int at = tiles.at(j), half = (j & 1) * SIZE;
        __syncthreads();
        const bool bad = __builtin_amdgcn_readfirstlane(spoilt[j & 1]) == j + 1, skip = bad || none(at);
        left_out |= bad;
        if (!skip) weigh(at, keys + half, values + half, std::false_type());
        if (j + 1 < until) store(j + 1, std::false_type());
        if (j + 2 < until) load(j + 2);
        if (!skip) product_along_rows<X, D, N / X::STEP, WHOLE>(lane, keys + half, terms, acc, A.K);
    }
    if (left_out) {
#pragma unroll 1
        for (int j = begin; j < until; ++j) {
            const int at = tiles.at(j);
            E *tile = keys + (j & 1) * SIZE;
            __syncthreads();
            load(j);
            store(j, std::true_type());
            __syncthreads();
            if (spoilt[j & 1] != j + 1) continue;
            const bool skip = none(at);
            if (!skip) weigh(at, tile, values + (j & 1) * SIZE, std::true_type());
            leave_finite<X, D, N, kWindowThreads>(tile);
            if (!skip) product_along_rows<X, D, N / X::STEP, WHOLE>(lane, tile, terms, acc, A.K);
            add_not_finite<X, D, N, kWindowThreads, true>(lane, tile, k + at * A.ks[1], A.ks[1], A.K, p.n - at, skip, acc, [&](int r) { return seen(line, at + r); });
        }
    }
    if (there && A.splits > 1) store_line<X, D>(A.pieces + (((p.b * A.heads + p.head) * A.splits + p.split) * A.T + line) * A.K, A.K, lane, acc, A.scale * scale.back());
    else if (there) store_line<X, D>(out + line * out_stride, A.K, lane, acc, A.scale * scale.back());
    if (hi < end && p.split == 0) zero_rows(out, out_stride, A.K, hi, end);
}

// ---------------------------------------------------------------- pieces of the keys
// Joins the pieces of queries that were cut along their keys (by the rule in sig_window.hip), in their order: outputs with the statistics and the rest, each piece's sums scaled
// to the largest maximum, or (GRADIENT) the queries' gradients.  Bound by memory: each piece is read once.  `lanes` threads (a power of two) take a token of a head, four columns each.
template <typename T, bool GRADIENT>
__global__ __launch_bounds__(kWindowThreads) void sig_window_join_pieces_kernel(WindowArgs A, int lanes)
{
    const int64_t id = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kWindowThreads / lanes) + threadIdx.x / lanes, line = id / A.T;
    const int token = (int)(id % A.T), dim = GRADIENT ? A.K : A.V, width = GRADIENT ? A.K : A.V + 2, c = threadIdx.x % lanes * 4;
    if (line >= A.B * A.heads) return;
    const int64_t b = line / A.heads, n = A.lengths ? A.lengths[b] : A.T, apart = (int64_t)A.T * width;
    if (token >= n || c >= dim) return;      // (behind the sequence there are zeros by now)
    const float *pieces = A.pieces + (line * A.splits * A.T + token) * width;
    float top = -INFINITY, total = 0.0f, x[4] = {};
    if (!GRADIENT)
        for (int i = 0; i < A.splits; ++i) top = fmaxf(top, pieces[i * apart + A.V]);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
    for (int i = 0; i < A.splits; ++i) {
        const float *piece = pieces + i * apart;
        float share = 1.0f;
        if (!GRADIENT) {
            share = __builtin_amdgcn_exp2f(piece[A.V] - base);
            total = fmaf(piece[A.V + 1], share, total);
        }
        if (c + 4 <= dim) {
            const Pack<float, 4> four = load_pack<float, 4>(piece + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(four.v[j], share, x[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < dim) x[j] = fmaf(piece[c + j], share, x[j]);
        }
    }
    const float r = GRADIENT ? 1.0f : 1.0f / total;
    const int64_t row = ((b * A.T + token) * A.heads + line % A.heads) * dim + c;
    T *to = (T *)(GRADIENT ? A.grad_q : A.out) + row;
    Pack<T, 4> four;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[j] *= r;
        four.v[j] = from_float<T>(x[j]);
    }
    const bool whole = c + 4 <= dim;
    if (whole) {
        store_pack(to, four);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < dim) to[j] = four.v[j];
    }
    if constexpr (!GRADIENT) {
        if (sizeof(T) == 2 && A.rest) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] -= to_float(four.v[j]);
            const unsigned rest = rest_of(x[2], x[3], rest_of(x[0], x[1], 0, false), true);
            if (whole) {
                store_pack(A.rest + row, __builtin_bit_cast(Pack<Rest, 4>, rest));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < dim) A.rest[row + j] = (Rest)(rest >> (8 * j));
            }
        }
        if (A.stats && c == 0) A.stats[line * A.T + token] = make_float2(base, r);
    }
}

// ---------------------------------------------------------------- gradient of keys and values
// Own lines are keys; queries and upstream gradients of all heads that share them come as tiles, one head after the other, so that the sum over these
// heads is one of registers.  Two wavefronts, on the same matrix unit, share M keys: the first holds the keys, works out p and adds up grad v; the second holds the
// values, takes p from LDS a tile later, and adds up grad k.  Each has half of the registers' load, and one multiplies while the other one
// does not (both gradients in one wavefront, one a unit: 1,510 us where this takes 1,190; 8 x 4,096 tokens, 16 heads of 128 bfloat16, window 1,024).  Few
// tiles, and those of the first tokens, which every query sees, are cut into parts along the queries, and joined from scratch.
constexpr int kKeyThreads = 2 * kWindowThreads;

template <typename T, typename X, int D, int N, bool WHOLE>
__global__ __launch_bounds__(kKeyThreads, 2) void sig_window_key_gradient_kernel(WindowArgs A)
{
    using E = typename X::E;
    constexpr int M = X::M, ROWS = kWindowWaves * M, QUERIES = N / M, STEPS = D / X::STEP, OUT = D / M, SIZE = N * X::template Tile<D>::PITCH, NUMBERS = QUERIES * X::REGS;
    constexpr float LIFT = std::is_same_v<E, f16> ? 32768.0f : 1.0f;      // of the probabilities, which are at most 1 (what float16 holds is small)
    __shared__ __attribute__((aligned(16))) E queries[3 * SIZE];
    __shared__ __attribute__((aligned(16))) E upstream[3 * SIZE];
    __shared__ __attribute__((aligned(16))) float most[3 * N], inverse[3 * N], delta[3 * N];
    __shared__ __attribute__((aligned(16))) f4 passed[2][kWindowWaves][NUMBERS / 4][64];      // p, as the lanes hold it
    __shared__ int spoilt[3];
    // which head and keys: the cut tiles' parts first, then the other tiles
    const int shared_heads = A.heads / A.group, pieces = A.cut * A.parts + A.tiles - A.cut;
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, lines = A.B * shared_heads;
    if (id >= lines * pieces) return;
    const bool by_eight = lines % 8 == 0;      // (see window_place)
    const int64_t head_line = by_eight ? id / 8 / pieces * 8 + id % 8 : id % lines;
    const int piece = (int)(by_eight ? id / 8 % pieces : id / lines);
    const int64_t b = head_line / shared_heads;
    const int shared = (int)(head_line % shared_heads), cut_pieces = A.cut * A.parts;
    const int tile = piece < cut_pieces ? piece / A.parts : piece - cut_pieces + A.cut, parts = piece < cut_pieces ? A.parts : 1, part = parts == 1 ? 0 : piece % A.parts;
    const int64_t counted = A.lengths ? A.lengths[b] : A.T;
    const int n = counted < 0 ? 0 : counted > A.T ? A.T : (int)counted;

    const int lane = threadIdx.x % 64, lo = tile * ROWS, end = min(lo + ROWS, A.T);
    T *out_k = (T *)A.grad_k + ((b * A.T) * shared_heads + shared) * A.K, *out_v = (T *)A.grad_v + ((b * A.T) * shared_heads + shared) * A.V;
    const int64_t k_stride = (int64_t)shared_heads * A.K, v_stride = (int64_t)shared_heads * A.V, g_stride = (int64_t)A.heads * A.V;
    const bool zeros = part == 0;      // whether this workgroup clears what stands behind the sequence
    if (lo >= n) {
        if (!zeros) return;
        zero_rows<kKeyThreads>(out_k, k_stride, A.K, lo, end);
        zero_rows<kKeyThreads>(out_v, v_stride, A.V, lo, end);
        return;
    }
    const int hi = min(end, n), wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64), pair = wave % kWindowWaves;
    const bool second = wave >= kWindowWaves;
    const int own = lo + pair * M, line = own + lane % M;
    const bool there = line < n;
    typename X::Frag held[STEPS];      // keys, or values
    {
        const int row = there ? line : lo;
        if (second) fragments_of<X, STEPS>(held, lane, (const T *)A.v + b * A.vs[0] + row * A.vs[1] + shared * A.vs[2], A.V, there, false);
        else fragments_of<X, STEPS>(held, lane, (const T *)A.k + b * A.ks[0] + row * A.ks[1] + shared * A.ks[2], A.K, there, A.negated);
    }
    const Seen seen = {A.window, A.sinks};
    // queries from lo on; where no key is one of the first tokens, those that have the last one in their window
    const int last = (lo < A.sinks ? n : (int)min((int64_t)n, (int64_t)hi - 1 + A.window)) - 1, all_tiles = last / N - lo / N + 1;
    // tiles of queries, of one head after the other: first ... first + tiles - 1, and of those numbers `from` to `until`
    int first = lo / N, tiles = all_tiles, from = 0, until = tiles * A.group;
    if (parts > 1 && A.even) {
        from = (int)((int64_t)tiles * A.group * part / parts);
        until = (int)((int64_t)tiles * A.group * (part + 1) / parts);
    } else if (parts > 1) {
        // (part 0 are the queries that have keys of this tile in their window, the others see the first tokens alone)
        const int near = ((int)min((int64_t)n, (int64_t)hi - 1 + A.window) - 1) / N - lo / N + 1, far = all_tiles - near;
        const int low = part == 0 ? 0 : near + (int)((int64_t)far * (part - 1) / (parts - 1)), high = part == 0 ? near : near + (int)((int64_t)far * part / (parts - 1));
        first += low;
        tiles = high - low;
        until = tiles * A.group;
    }
    const int count = until - from;
    struct Place { int head, at; };      // of a tile of queries
    auto next = [&](Place &w) {
        w.at += N;
        if (w.at >= (first + tiles) * N) {
            w.at = first * N;
            ++w.head;
        }
    };
    TileMover<T, X, D, N, kKeyThreads, WHOLE> query_tile, upstream_tile;
    float2 stats_tile;
    float delta_tile;
    auto load = [&](const Place &w) {
        const int head = shared * A.group + w.head;
        query_tile.load((const T *)A.q + b * A.qs[0] + head * A.qs[2] + w.at * A.qs[1], A.qs[1], A.K, n - w.at);
        upstream_tile.load((const T *)A.grad_out + ((b * A.T + w.at) * A.heads + head) * A.V, g_stride, A.V, n - w.at);
        stats_tile = make_float2(0.0f, 0.0f);
        delta_tile = 0.0f;
        if (threadIdx.x < N && w.at + (int)threadIdx.x < n) {
            const int64_t place = (b * A.heads + head) * A.T + w.at + threadIdx.x;
            stats_tile = A.stats[place];
            delta_tile = A.delta[place];
        }
    };
    // `room`: of three, j % 3
    auto store = [&](const Place &w, int j, int room, auto careful) {
        constexpr bool NANS = decltype(careful)::value;
        query_tile.template store<NANS>(queries + room * SIZE, A.K, n - w.at);
        upstream_tile.store(upstream + room * SIZE, A.V, n - w.at);
        if (threadIdx.x < N) {
            most[room * N + threadIdx.x] = stats_tile.x;
            inverse[room * N + threadIdx.x] = stats_tile.y;
            delta[room * N + threadIdx.x] = delta_tile;
        }
        if (!seen.all(w.at, w.at + N - 1, lo, lo + ROWS - 1) && (query_tile.spoilt(A.K, n - w.at) || upstream_tile.spoilt(A.V, n - w.at))) spoilt[room] = j + 1;
    };
    typename X::Result acc[OUT] = {};
    TermScale scale;
    typename X::Frag weights[N / X::STEP];
    auto hidden = [&](int at) { return at + N > n || !seen.all(at, at + N - 1, own, own + M - 1); };
    auto sees = [&](int query) { return (query < n) & seen(query, line); };
    // the probabilities of a tile, for the second wavefront too
    auto weigh_values = [&](int at, int room, int half, auto careful) {
        typename X::Result s[QUERIES] = {};
        product_of_rows<X, D, QUERIES, WHOLE, 4>(lane, queries + room * SIZE, held, s, A.K);
        if constexpr (decltype(careful)::value) settle_infinities<X, D, QUERIES>(lane, queries + room * SIZE, held, s);
#pragma unroll
        for (int t = 0; t < QUERIES; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; i += 4) {
                const int row = room * N + t * M + X::row_of(lane, i);
                const f4 x = *(const f4 *)(most + row), r = *(const f4 *)(inverse + row);
#pragma unroll
                for (int c = 0; c < 4; ++c) s[t][i + c] = __builtin_amdgcn_exp2f(fmaf(s[t][i + c], A.power, -x[c])) * r[c];
            }
        if (hidden(at)) {
#pragma unroll
            for (int t = 0; t < QUERIES; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) s[t][i] = sees(at + t * M + X::row_of(lane, i)) ? s[t][i] : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < QUERIES; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; i += 4) passed[half][pair][(t * X::REGS + i) / 4][lane] = f4{s[t][i], s[t][i + 1], s[t][i + 2], s[t][i + 3]};
        if constexpr (std::is_same_v<E, f16>) {
#pragma unroll
            for (int t = 0; t < QUERIES; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) s[t][i] *= LIFT;
        }
        // (rounded for their product, as in the forward pass; the second wavefront has them in float32, and rounds its terms)
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) weights[step] = X::of_results(s, step);
    };
    auto weigh_keys = [&](int at, int room, int half) {
        typename X::Result u[QUERIES] = {};
        product_of_rows<X, D, QUERIES, WHOLE, 4>(lane, upstream + room * SIZE, held, u, A.V);
#pragma unroll
        for (int t = 0; t < QUERIES; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; i += 4) {
                const f4 p = passed[half][pair][(t * X::REGS + i) / 4][lane], d = *(const f4 *)(delta + room * N + t * M + X::row_of(lane, i));
#pragma unroll
                for (int c = 0; c < 4; ++c) u[t][i + c] = p[c] * (u[t][i + c] - d[c]);
            }
        if (hidden(at)) {
#pragma unroll
            for (int t = 0; t < QUERIES; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) u[t][i] = sees(at + t * M + X::row_of(lane, i)) ? u[t][i] : 0.0f;
        }
        if constexpr (std::is_same_v<E, f16>) {
            float shrink;
            if (scale.grown<M, QUERIES>(u, &shrink)) {
#pragma unroll
                for (int t = 0; t < OUT; ++t)
#pragma unroll
                    for (int i = 0; i < X::REGS; ++i) acc[t][i] *= shrink;
            }
#pragma unroll
            for (int t = 0; t < QUERIES; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) u[t][i] *= scale.factor;
        }
#pragma unroll
        for (int step = 0; step < N / X::STEP; ++step) weights[step] = X::of_results(u, step);
    };
    auto none = [&](int at) { return own >= hi || seen.none(at, min(at + N, n) - 1, own, min(own + M, hi) - 1); };
    bool all_bad = false;      // (infinite keys, whose products with parts are no numbers)
    if constexpr (X::PLANES > 1) all_bad = __syncthreads_or(!second && any_infinite<STEPS>(held));
    // Tile j is the first wavefronts' and tile j - 1 the second ones', tile j + 1 goes to LDS, j + 2 is on its way
    bool left_out = false, skipped = true;      // skipped: the tile before
    if (threadIdx.x < 3) spoilt[threadIdx.x] = 0;
    const Place begin = {tiles > 0 ? from / tiles : 0, (first + (tiles > 0 ? from % tiles : 0)) * N};
    Place now = begin, before = now, ahead = now;
    if (count > 0) load(ahead);
    __syncthreads();
    if (count > 0) store(ahead, 0, 0, std::false_type());
    next(ahead);
    if (count > 1) load(ahead);
    int room = 0, behind = 2;
    for (int j = 0; j <= count; ++j) {
        const int following = room == 2 ? 0 : room + 1;
        __syncthreads();
        const bool bad = j < count && (all_bad || __builtin_amdgcn_readfirstlane(spoilt[room]) == j + 1), skip = bad || j == count || none(now.at);
        left_out |= bad;
        if (!second && !skip) {
            weigh_values(now.at, room, j & 1, std::false_type());
            product_along_rows<X, D, N / X::STEP, WHOLE, 2>(lane, upstream + room * SIZE, weights, acc, A.V);
        }
        if (second && !skipped) {
            weigh_keys(before.at, behind, ~j & 1);
            product_along_rows<X, D, N / X::STEP, WHOLE, 2>(lane, queries + behind * SIZE, weights, acc, A.K);
        }
        if (j + 1 < count) store(ahead, j + 1, following, std::false_type());
        next(ahead);
        if (j + 2 < count) load(ahead);
        skipped = skip;
        before = now;
        next(now);
        behind = room;
        room = following;
    }
    if (left_out) {
        now = begin;
#pragma unroll 1
        for (int j = 0; j < count; ++j, next(now)) {
            const int at = now.at, head = shared * A.group + now.head;
            __syncthreads();
            load(now);
            store(now, j, 0, std::true_type());
            __syncthreads();
            if (!all_bad && spoilt[0] != j + 1) continue;
            const bool skip = none(at);
            if (!second && !skip) weigh_values(at, 0, 0, std::true_type());
            __syncthreads();
            if (second && !skip) weigh_keys(at, 0, 0);
            leave_finite<X, D, N, kKeyThreads>(queries);
            leave_finite<X, D, N, kKeyThreads>(upstream);
            if (!second && !skip) product_along_rows<X, D, N / X::STEP, WHOLE, 2>(lane, upstream, weights, acc, A.V);
            if (second && !skip) product_along_rows<X, D, N / X::STEP, WHOLE, 2>(lane, queries, weights, acc, A.K);
            add_not_finite<X, D, N, kKeyThreads, false>(lane, upstream, (const T *)A.grad_out + ((b * A.T + at) * A.heads + head) * A.V, g_stride, A.V, n - at,
                                                        skip || second, acc, [&](int r) { return sees(at + r); });
            add_not_finite<X, D, N, kKeyThreads, true>(lane, queries, (const T *)A.q + b * A.qs[0] + head * A.qs[2] + at * A.qs[1], A.qs[1], A.K, n - at,
                                                       skip || !second, acc, [&](int r) { return sees(at + r); });
        }
    }
    const float own_scale = second ? A.scale * scale.back() : 1.0f / LIFT;
    if (there && (parts == 1 || (part == 0 && line >= A.joined))) {
        if (second) store_line<X, D>(out_k + line * k_stride, A.K, lane, acc, own_scale);
        else store_line<X, D>(out_v + line * v_stride, A.V, lane, acc, own_scale);
    } else if (there && line < A.joined) {
        float *to = A.sums + (((head_line * A.cut + tile) * parts + part) * ROWS + (line - lo)) * (A.K + A.V);
        if (second) store_line<X, D>(to, A.K, lane, acc, own_scale);
        else store_line<X, D>(to + A.K, A.V, lane, acc, own_scale);
    }
    if (hi < end && zeros) {
        zero_rows<kKeyThreads>(out_k, k_stride, A.K, hi, end);
        zero_rows<kKeyThreads>(out_v, v_stride, A.V, hi, end);
    }
}

// The sums of cut tiles' parts, in their order: some tokens a workgroup, `lanes` threads (a power of two) each
template <typename T, int ROWS>
__global__ __launch_bounds__(kWindowThreads) void sig_window_join_kernel(WindowArgs A, int lanes)
{
    const int shared_heads = A.heads / A.group, width = A.K + A.V;
    const int64_t id = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kWindowThreads / lanes) + threadIdx.x / lanes, head_line = id / A.joined;
    const int key = (int)(id % A.joined);
    if (head_line >= A.B * shared_heads) return;
    const int64_t b = head_line / shared_heads, n = A.lengths ? A.lengths[b] : A.T;
    if (key >= n || key >= A.T) return;      // (those are zero by now)
    const float *sums = A.sums + ((head_line * A.cut + key / ROWS) * A.parts * ROWS + key % ROWS) * width;
    for (int c = threadIdx.x % lanes; c < width; c += lanes) {
        float sum = 0.0f;
#pragma unroll 8
        for (int i = 0; i < A.parts; ++i) sum += sums[(int64_t)i * ROWS * width + c];
        const int64_t row = (b * A.T + key) * shared_heads + head_line % shared_heads;
        if (c < A.K) ((T *)A.grad_k)[row * A.K + c] = from_float<T>(sum);
        else ((T *)A.grad_v)[row * A.V + c - A.K] = from_float<T>(sum);
    }
}

// ---------------------------------------------------------------- launches
enum WindowPass { WINDOW_FORWARD, WINDOW_QUERY_GRADIENT, WINDOW_KEY_GRADIENT };

hipError_t launch_window_f32(const WindowArgs &A, WindowPass pass, hipStream_t st);
hipError_t launch_window_bf16(const WindowArgs &A, WindowPass pass, hipStream_t st);
hipError_t launch_window_f16(const WindowArgs &A, WindowPass pass, hipStream_t st);

// Whether float32 is multiplied as three parts (SplitTiles), with rows of up to 64 components or of 96 that are all there
constexpr bool window_splits(int K, int V) { return (K > V ? K : V) <= 64 || (K == 96 && V == 96); }

// lines of a workgroup
inline int window_rows(int type, int K, int V) { return kWindowWaves * ((type == SIG_F32 ? !window_splits(K, V) : (K > V ? K : V) > 128) ? 16 : 32); }

inline dim3 window_grid(int64_t blocks)
{
    const int64_t across = ((int64_t)1 << 32) / (2 * kWindowThreads) - 1;      // (a launch holds fewer than 2^32 threads along an axis)
    return dim3((unsigned)(blocks < across ? blocks : across), (unsigned)((blocks + across - 1) / across));
}

template <typename T>
hipError_t launch_window(const WindowArgs &A, WindowPass given, hipStream_t st)
{
    const int dim = A.K > A.V ? A.K : A.V;
    const int64_t shared = A.B * (A.heads / A.group);
    auto go = [&](auto d, auto whole, auto pass) {
        constexpr int D = decltype(d)::value;
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr WindowPass PASS = decltype(pass)::value;
        constexpr bool SPLIT = sizeof(T) == 4 && (WHOLE ? window_splits(D, D) : D <= 64);
        using X = std::conditional_t<SPLIT, SplitTiles, std::conditional_t<(D > 128), SmallTiles<T>, Tiles<T>>>;
        // tokens of a tile
        constexpr int BYTES = D * (int)sizeof(T), ROWS = kWindowWaves * X::M;
        constexpr int N = BYTES > 512 ? 16 : sizeof(T) == 4 || BYTES > (PASS == WINDOW_FORWARD && WHOLE ? 256 : 128) ? 32 : 64;
        if constexpr (PASS != WINDOW_KEY_GRADIENT) {
            constexpr bool GRADIENT = PASS == WINDOW_QUERY_GRADIENT;
            const dim3 grid = window_grid(A.B * A.heads * A.tiles * A.splits);
            if constexpr (GRADIENT) sig_window_query_gradient_kernel<T, X, D, N, WHOLE><<<grid, kWindowThreads, 0, st>>>(A);
            else sig_window_forward_kernel<T, X, D, N, WHOLE><<<grid, kWindowThreads, 0, st>>>(A);
            if (A.splits > 1) {
                int lanes = 1;
                while (lanes * 4 < (GRADIENT ? A.K : A.V)) lanes *= 2;
                const int at_once = kWindowThreads / lanes;
                sig_window_join_pieces_kernel<T, GRADIENT><<<window_grid((A.B * A.heads * A.T + at_once - 1) / at_once), kWindowThreads, 0, st>>>(A, lanes);
            }
        } else {
            const int64_t pieces = A.cut * A.parts + A.tiles - A.cut;
            sig_window_key_gradient_kernel<T, X, D, N, WHOLE><<<window_grid(shared * pieces), kKeyThreads, 0, st>>>(A);
            if (A.parts > 1) {
                int lanes = 64;
                while (lanes < A.K + A.V && lanes < kWindowThreads) lanes *= 2;
                const int at_once = kWindowThreads / lanes;
                sig_window_join_kernel<T, ROWS><<<window_grid((shared * A.joined + at_once - 1) / at_once), kWindowThreads, 0, st>>>(A, lanes);
            }
        }
    };
    auto of = [&](auto d, auto whole) {
        if (given == WINDOW_FORWARD) go(d, whole, std::integral_constant<WindowPass, WINDOW_FORWARD>());
        else if (given == WINDOW_QUERY_GRADIENT) go(d, whole, std::integral_constant<WindowPass, WINDOW_QUERY_GRADIENT>());
        else go(d, whole, std::integral_constant<WindowPass, WINDOW_KEY_GRADIENT>());
    };
    auto with = [&](auto d) {
        if (A.K == decltype(d)::value && A.V == A.K) of(d, std::true_type());
        else of(d, std::false_type());
    };
    // (rows of 129 to 192 components in their own instance instead of that of 256: 4 x 2,048 tokens, 16 heads (4 shared) of 192 bfloat16 forward 682 -> 247 us, with the gradient
    // 2,122 -> 1,071; 1 x 1,035, 80 heads (10 shared) of 80 x 130 float16 1,187 -> 925; 4 x 1,000, 8 heads of 192 float32 1,206 -> 985)
    if (dim <= 32) with(std::integral_constant<int, 32>());
    else if (dim <= 64) with(std::integral_constant<int, 64>());
    else if (dim <= 96) with(std::integral_constant<int, 96>());
    else if (dim <= 128) with(std::integral_constant<int, 128>());
    else if (dim <= 192) with(std::integral_constant<int, 192>());
    else with(std::integral_constant<int, 256>());
    return hipGetLastError();
}

}  // namespace sig
#endif
