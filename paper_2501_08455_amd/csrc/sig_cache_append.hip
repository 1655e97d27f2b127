// Keys and values of new tokens into a paged cache, keys turned by their positions on the way, and the tokens' queries turned (include/sig_sequence.h).
//
// Bound by memory: each value is read and written once.  A workgroup takes a few tokens, works out their cosines and sines once for all
// heads, in LDS, and walks over the lines (a token's head of q, k or v), several loads in flight a thread.  Into pages of 8 bits: a workgroup
// takes a page's tokens of one head, since they share a scale, which is known when all of them have been read; more than a thread's worth each are
// read twice.
#include <type_traits>

#include "sig_cache.h"
#include "sig_context.h"
#include "sig_turn.h"

using namespace sig;

namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 16;      // of a workgroup
constexpr int kTable = 2048;         // pairs of a workgroup's tokens

template <typename T>
constexpr int kGroup = 16 / sizeof(T);     // values of the widest load

struct AppendArgs {
    CacheArgs cache;
    const void *q, *k, *v;
    void *q_out;
    int64_t qs[3], ks[3], vs[3], ps[2];     // strides: batch, token, head
    int64_t B, T;
    int heads;                               // of q
    const int64_t *lengths, *counts;
    const void *positions;
    int position_type;
    const double *frequencies;
    int turned;
    float scale;
    int tokens, places;                      // of a workgroup; threads of a line, a power of two
    int64_t token_blocks;                    // workgroups of whole tokens; behind them those of pages
    int pages;                               // that a sequence's new tokens may touch
};

__device__ int64_t held_by(const AppendArgs &A, int64_t b)
{
    const int64_t n = A.lengths[b], most = (int64_t)1 << 62;
    return n < 0 ? 0 : n > most ? most : n;
}

__device__ int64_t new_of(const AppendArgs &A, int64_t b)
{
    const int64_t n = A.counts ? A.counts[b] : A.T;
    return n < 0 ? 0 : n > A.T ? A.T : n;
}

__device__ double position_of(const AppendArgs &A, int64_t b, int64_t t, int64_t place)
{
    return A.positions ? position_at(A.positions, A.position_type, b * A.ps[0] + t * A.ps[1]) : (double)place;
}

// N values of a turned line, or N pairs in the half layout; M values of a copied one.  How the components are laid out over units (see sig_rotary.hip):
// turned units first, then the copied ones, the last of which ends with the line
template <typename T, int N, bool INTERLEAVED>
struct Line {
    static constexpr int M = kGroup<T>;
    int dim, turned;
    __device__ int turned_units() const { return INTERLEAVED ? turned / N : turned / 2 / N; }
    __device__ int units() const { return turned_units() + (dim - turned + M - 1) / M; }
    __device__ bool copied(int unit) const { return unit >= turned_units(); }
    __device__ bool few() const { return dim - turned < M; }      // (of the copied ones: fewer than a unit)
    __device__ int at(int unit) const { return !copied(unit) ? unit * N : few() ? turned : min(turned + (unit - turned_units()) * M, dim - M); }
};

// (a, b) of each of the pairs of a turned unit, with the angles of its token
template <typename T, int N, bool INTERLEAVED>
__device__ void turn_unit(float *low, float *high, const float2 *angles, int at)
{
    if constexpr (INTERLEAVED) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            const float2 turn = angles[at / 2 + j / 2];
            const float a = low[j], b = low[j + 1];
            low[j] = a * turn.x - b * turn.y;
            low[j + 1] = a * turn.y + b * turn.x;
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float2 turn = angles[at + j];
            const float a = low[j], b = high[j];
            low[j] = a * turn.x - b * turn.y;
            high[j] = a * turn.y + b * turn.x;
        }
    }
}

// N values on their way, as the words that hold them where they are whole words
template <typename T, int N>
using Held = std::conditional_t<(N * sizeof(T) >= 4), Words<T, (N * sizeof(T) >= 4 ? N : 4)>, Pack<T, N>>;

template <typename T, int N>
__device__ inline Held<T, N> load_held(const T *from)
{
    return __builtin_bit_cast(Held<T, N>, load_pack<T, N>(from));
}

template <typename T, int N>
__device__ inline void floats_of(const Held<T, N> &held, float *x)
{
    const auto values = __builtin_bit_cast(Pack<T, N>, held);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = to_float(values.v[j]);
}

template <typename T, int N>
__device__ inline void store_floats(T *to, const float *x)
{
    Pack<T, N> values;
#pragma unroll
    for (int j = 0; j < N; ++j) values.v[j] = from_float<T>(x[j]);
    store_pack(to, values);
}

// Whole tokens: all lines of q, and those of k and v where the cache has their type
template <typename T, int N, bool INTERLEAVED, bool WIDE>
__device__ void append_tokens(const AppendArgs &A, int64_t block, float2 *table)
{
    constexpr int AT_ONCE = 4;
    constexpr int M = kGroup<T>;
    struct Token {
        int64_t from[3], to[3];      // of q, k and v: in values, the first head's
        int live, written;           // whether the token is there, and its place has a page
    };
    __shared__ Token of[kMostTokens];
    const int half = A.turned / 2, G = WIDE ? A.cache.heads : 0, lines = A.heads + 2 * G;
    const int64_t first = block * A.tokens, all = A.B * A.T;
    const int tokens = all - first < A.tokens ? (int)(all - first) : A.tokens;
    for (int i = threadIdx.x; i < tokens * half || i < tokens; i += kThreads) {
        if (i < tokens) {
            const int64_t b = (first + i) / A.T, t = (first + i) % A.T, place = held_by(A, b) + t;
            Token token;
            token.live = t < new_of(A, b);
            const int64_t page = WIDE && token.live ? A.cache.page_of(b, place / A.cache.page_tokens) : -1, slot = place % A.cache.page_tokens;
            token.written = page >= 0;
            token.from[0] = b * A.qs[0] + t * A.qs[1];
            token.from[1] = b * A.ks[0] + t * A.ks[1];
            token.from[2] = b * A.vs[0] + t * A.vs[1];
            token.to[0] = (first + i) * A.heads * A.cache.K;
            token.to[1] = page * A.cache.keys.page + slot * A.cache.keys.slot;
            token.to[2] = page * A.cache.values.page + slot * A.cache.values.slot;
            of[i] = token;
        }
        if (i < tokens * half) {
            const int64_t b = (first + i / half) / A.T, t = (first + i / half) % A.T;
            float c, s;
            turn(position_of(A, b, t, held_by(A, b) + t), A.frequencies[i % half], &c, &s);
            table[i] = make_float2(A.scale * c, A.scale * s);
        }
    }
    __syncthreads();
    const Line<T, N, INTERLEAVED> turned_line = {A.cache.K, A.turned}, copied_line = {A.cache.V, 0};
    const int turned_units = turned_line.units(), copied_units = copied_line.units(), most = max(turned_units, G ? copied_units : 0);
    const int apart = kThreads / A.places, token_step = apart / lines, line_step = apart % lines;
    for (int unit = threadIdx.x % A.places; unit < most; unit += A.places) {
        const int turned_at = turned_line.at(unit), copied_at = copied_line.at(unit);
        // what the unit is in lines of q and k: 1 turned, 2 copied, 3 fewer than a unit, 0 nothing; and of v: 2, 3, 0
        const int turned_what = unit >= turned_units ? 0 : !turned_line.copied(unit) ? 1 : turned_line.few() ? 3 : 2;
        const int copied_what = unit >= copied_units ? 0 : copied_line.few() ? 3 : 2;
        int token = threadIdx.x / A.places / lines, line = threadIdx.x / A.places % lines;
        while (token < tokens) {
            Held<T, M> same[AT_ONCE];
            Held<T, N> low[AT_ONCE], high[AT_ONCE];
            const T *source[AT_ONCE];
            T *to[AT_ONCE];
            int tokens_of[AT_ONCE], what[AT_ONCE], widths[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                what[i] = 0;
                tokens_of[i] = token;
                if (token < tokens) {
                    const Token &its = of[token];
                    const bool is_query = line < A.heads, is_value = line >= A.heads + G;
                    const int head = is_query ? line : is_value ? line - A.heads - G : line - A.heads;
                    what[i] = is_value ? copied_what : turned_what;
                    if (!is_query && !its.written) what[i] = 0;
                    const int at = is_value ? copied_at : turned_at;
                    widths[i] = is_value ? A.cache.V : A.cache.K - A.turned;
                    source[i] = (is_query ? (const T *)A.q + its.from[0] + head * A.qs[2] : is_value ? (const T *)A.v + its.from[2] + head * A.vs[2]
                                                                                                    : (const T *)A.k + its.from[1] + head * A.ks[2]) + at;
                    to[i] = (is_query ? (T *)A.q_out + its.to[0] + (int64_t)head * A.cache.K : is_value ? (T *)A.cache.values.values + its.to[2] + head * A.cache.values.head
                                                                                                      : (T *)A.cache.keys.values + its.to[1] + head * A.cache.keys.head) + at;
                    if (its.live) {
                        if (what[i] == 2) same[i] = load_held<T, M>(source[i]);
                        if (what[i] == 1) {
                            low[i] = load_held<T, N>(source[i]);
                            if (!INTERLEAVED) high[i] = load_held<T, N>(source[i] + half);
                        }
                    } else {
                        what[i] = -what[i];      // (zeros)
                    }
                }
                token += token_step;
                line += line_step;
                if (line >= lines) {
                    line -= lines;
                    ++token;
                }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (what[i] == 1) {
                    float a[N], b[N];
                    floats_of<T, N>(low[i], a);
                    if (!INTERLEAVED) floats_of<T, N>(high[i], b);
                    turn_unit<T, N, INTERLEAVED>(a, b, table + tokens_of[i] * half, turned_at);
                    store_floats<T, N>(to[i], a);
                    if (!INTERLEAVED) store_floats<T, N>(to[i] + half, b);
                } else if (what[i] == 2) {
                    store_pack(to[i], __builtin_bit_cast(Pack<T, M>, same[i]));
                } else if (what[i] == -1) {
                    const float none[N] = {};
                    store_floats<T, N>(to[i], none);
                    if (!INTERLEAVED) store_floats<T, N>(to[i] + half, none);
                } else if (what[i] == -2) {
                    const float none[M] = {};
                    store_floats<T, M>(to[i], none);
                } else if (what[i] != 0) {
                    for (int j = 0; j < widths[i]; ++j) to[i][j] = what[i] > 0 ? source[i][j] : from_float<T>(0.0f);
                }
            }
        }
    }
}

constexpr float kLeastScale = 0x1p-126f;

// the smallest power of two, 2^-126 at least, that is no less than most / 448
__device__ inline float narrow_scale(float most)
{
    const float ratio = most / kMostNarrow;
    const unsigned bits = __builtin_bit_cast(unsigned, ratio);
    if (ratio <= kLeastScale) return kLeastScale;
    return __builtin_bit_cast(float, (bits + 0x7fffffu) & 0x7f800000u);
}

// A page's new tokens of one head, into 8 bits.  `block` counts sequences, pages that they may touch, heads, and keys and values
template <typename T, int N, bool INTERLEAVED>
__device__ void append_page(const AppendArgs &A, int64_t block, float2 *table)
{
    constexpr int M = kGroup<T>;
    __shared__ float mosts[kThreads / 64];
    const bool is_value = block % 2;
    const int head = (int)(block / 2 % A.cache.heads);
    const int64_t number = block / 2 / A.cache.heads % A.pages, b = block / 2 / A.cache.heads / A.pages;
    const int64_t held = held_by(A, b), end = held + new_of(A, b), P = A.cache.page_tokens;
    const int64_t at_page = held / P + number, low_place = max(held, at_page * P), high_place = min(end, (at_page + 1) * P);
    if (low_place >= high_place) return;
    const int64_t page = A.cache.page_of(b, at_page);
    if (page < 0) return;
    const Pages &pages = is_value ? A.cache.values : A.cache.keys;
    const Line<T, N, INTERLEAVED> shape = {is_value ? A.cache.V : A.cache.K, is_value ? 0 : A.turned};
    const int half = shape.turned / 2, units = shape.units(), tokens = (int)(high_place - low_place), slot = (int)(low_place - at_page * P);
    const int64_t t0 = low_place - held;
    const T *source = is_value ? (const T *)A.v + b * A.vs[0] + t0 * A.vs[1] + head * A.vs[2] : (const T *)A.k + b * A.ks[0] + t0 * A.ks[1] + head * A.ks[2];
    const int64_t source_stride = is_value ? A.vs[1] : A.ks[1];
    Narrow *to = (Narrow *)pages.values + page * pages.page + head * pages.head;
    const int at_once = half ? min(tokens, kTable / half) : tokens;      // tokens whose angles the table holds
    // the cosines and sines of n tokens
    auto angles = [&](int first, int n) {
        if (!half) return;
        __syncthreads();
        for (int i = threadIdx.x; i < n * half; i += kThreads) {
            const int64_t t = t0 + first + i / half;
            float c, s;
            turn(position_of(A, b, t, held + t), A.frequencies[i % half], &c, &s);
            table[i] = make_float2(A.scale * c, A.scale * s);
        }
        __syncthreads();
    };
    // f(token, component, values, count) of all values as they are before they are rounded
    auto each = [&](auto f, bool again) {
        for (int first = 0; first < tokens; first += at_once) {
            const int n = min(at_once, tokens - first);
            if (!(again && at_once == tokens)) angles(first, n);
            for (int i = threadIdx.x; i < n * units; i += kThreads) {
                const int token = first + i / units, unit = i % units, at = shape.at(unit);
                const T *p = source + token * source_stride + at;
                if (!shape.copied(unit)) {
                    const Pack<T, N> low = load_pack<T, N>(p);
                    Pack<T, N> high = low;
                    if (!INTERLEAVED) high = load_pack<T, N>(p + half);
                    float x[N], y[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        x[j] = to_float(low.v[j]);
                        y[j] = to_float(high.v[j]);
                    }
                    turn_unit<T, N, INTERLEAVED>(x, y, table + (token - first) * half, at);
                    f(token, at, x, std::integral_constant<int, N>());
                    if (!INTERLEAVED) f(token, at + half, y, std::integral_constant<int, N>());
                } else if (shape.few()) {
                    for (int j = 0; j < shape.dim - shape.turned; ++j) {
                        float x[1] = {to_float(p[j])};
                        f(token, at + j, x, std::integral_constant<int, 1>());
                    }
                } else {
                    const Pack<T, M> same = load_pack<T, M>(p);
                    float x[M];
#pragma unroll
                    for (int j = 0; j < M; ++j) x[j] = to_float(same.v[j]);
                    f(token, at, x, std::integral_constant<int, M>());
                }
            }
        }
    };
    // (a value of each thread: it stays where it is until the scale is known)
    const bool one = tokens * units <= kThreads && at_once == tokens;
    const int own_token = threadIdx.x / units, own_unit = threadIdx.x % units, own_at = shape.at(own_unit);
    const int own = !one || own_token >= tokens ? 0 : !shape.copied(own_unit) ? 1 : shape.few() ? 3 : 2;
    float x[M > N ? M : N] = {}, y[N] = {};
    float most = 0.0f;
    auto larger = [&](const float *values, int n) {
#pragma unroll
        for (int j = 0; j < n; ++j) {
            const float size = fabsf(values[j]);
            most = size <= 3.4028234663852886e38f ? fmaxf(most, size) : most;
        }
    };
    const float before = pages.scales[page * A.cache.heads + head];
    if (one) {
        const T *p = source + own_token * source_stride + own_at;
        Held<T, N> low, high;
        if (own == 1) {
            low = load_held<T, N>(p);
            if (!INTERLEAVED) high = load_held<T, N>(p + half);
        } else if (own == 2) {
            floats_of<T, M>(load_held<T, M>(p), x);
        } else if (own == 3) {
            for (int j = 0; j < shape.dim - shape.turned; ++j) most = fabsf(to_float(p[j])) <= 3.4028234663852886e38f ? fmaxf(most, fabsf(to_float(p[j]))) : most;
        }
        angles(0, tokens);
        if (own == 1) {
            floats_of<T, N>(low, x);
            if (!INTERLEAVED) floats_of<T, N>(high, y);
            turn_unit<T, N, INTERLEAVED>(x, y, table + own_token * half, own_at);
            larger(x, N);
            if (!INTERLEAVED) larger(y, N);
        } else if (own == 2) {
            larger(x, M);
        }
    } else {
        each([&](int, int, const float *values, auto n) { larger(values, decltype(n)::value); }, false);
    }
#pragma unroll
    for (int i = 1; i < 64; i *= 2) most = fmaxf(most, __shfl_xor(most, i));
    if (threadIdx.x % 64 == 0) mosts[threadIdx.x / 64] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) most = fmaxf(most, mosts[i]);
    // (slot 0: the page keeps nothing from before)
    const float need = most > 0.0f ? narrow_scale(most) : slot == 0 ? 1.0f : kLeastScale, scale = slot == 0 ? need : fmaxf(need, before), inverse = 1.0f / scale;
    if (slot > 0 && scale > before) {
        const float shrink = before * inverse;
        for (int i = threadIdx.x; i < slot * shape.dim; i += kThreads) {
            Narrow *x = to + i / shape.dim * pages.slot + i % shape.dim;
            *x = to_narrow(from_narrow(*x) * shrink);
        }
    }
    if (threadIdx.x == 0) pages.scales[page * A.cache.heads + head] = scale;
    auto put = [&](int token, int at, const float *values, auto n) {
        constexpr int COUNT = decltype(n)::value;
        Pack<Narrow, COUNT> narrow;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) narrow.v[j] = to_narrow(values[j] * inverse);
        store_pack(to + (slot + token) * pages.slot + at, narrow);
    };
    if (!one) {
        each(put, true);
    } else if (own == 1) {
        put(own_token, own_at, x, std::integral_constant<int, N>());
        if (!INTERLEAVED) put(own_token, own_at + half, y, std::integral_constant<int, N>());
    } else if (own == 2) {
        put(own_token, own_at, x, std::integral_constant<int, M>());
    } else if (own == 3) {
        const T *p = source + own_token * source_stride + own_at;
        for (int j = 0; j < shape.dim - shape.turned; ++j) {
            const float value = to_float(p[j]);
            put(own_token, own_at + j, &value, std::integral_constant<int, 1>());
        }
    }
}

template <typename T, int N, bool INTERLEAVED, bool NARROW>
__global__ __launch_bounds__(kThreads) void sig_cache_append_kernel(AppendArgs A)
{
    __shared__ float2 table[kTable];
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (block < A.token_blocks) append_tokens<T, N, INTERLEAVED, !NARROW>(A, block, table);
    else if (NARROW && block - A.token_blocks < A.B * A.pages * A.cache.heads * 2) append_page<T, N, INTERLEAVED>(A, block - A.token_blocks, table);
}

}  // namespace

extern "C" int sig_cache_append(sig_ctx *ctx, const sig_cache_t *cache, const sig_append_t *shape, const void *q, const void *k, const void *v,
                                const int64_t *lengths, const int64_t *counts, void *q_out, void *hip_stream)
{
    if (!ctx || !shape) return SIG_ERR_INVALID;
    const sig_append_t &s = *shape;
    if (!valid_type(s.type) || !valid_cache(cache, s.type) || s.B < 0 || s.T < 0 || s.heads < 0 || s.turned < 0 || s.turned > cache->key_dim || s.turned % 2 ||
        (s.positions && (s.position_type < SIG_POSITION_I32 || s.position_type > SIG_POSITION_F64)))
        return SIG_ERR_INVALID;
    if (s.B == 0 || s.T == 0) return SIG_OK;
    if (!k || !v || !lengths || (s.heads && (!q || !q_out)) || (s.turned && !s.frequencies)) return SIG_ERR_INVALID;
    const int64_t lines = s.heads + 2 * (int64_t)cache->heads, widest = cache->key_dim > cache->value_dim ? cache->key_dim : cache->value_dim;
    if (s.B > INT32_MAX / s.T || lines > INT32_MAX / kMostTokens || widest * lines > INT32_MAX || cache->page_tokens > INT32_MAX / widest) return SIG_ERR_TOO_LARGE;
    if (s.turned / 2 > kTable) return SIG_ERR_UNSUPPORTED;
    AppendArgs A = {};
    A.cache = cache_arguments(*cache);
    A.q = q;
    A.k = k;
    A.v = v;
    A.q_out = q_out;
    for (int i = 0; i < 3; ++i) {
        A.qs[i] = s.q_strides[i];
        A.ks[i] = s.k_strides[i];
        A.vs[i] = s.v_strides[i];
    }
    A.ps[0] = s.position_strides[0];
    A.ps[1] = s.position_strides[1];
    A.B = s.B;
    A.T = s.T;
    A.heads = s.heads;
    A.lengths = lengths;
    A.counts = counts;
    A.positions = s.positions;
    A.position_type = s.position_type;
    A.frequencies = s.frequencies;
    A.turned = (int)s.turned;
    A.scale = (float)s.scale;
    const bool narrow = cache->type == SIG_E4M3;
    // tokens that share a workgroup: as many as leave eight workgroups a unit
    const int64_t share = s.B * s.T / (8 * (int64_t)ctx->num_cu), room = s.turned ? kTable / (s.turned / 2) : kMostTokens;
    A.tokens = (int)(share < 1 ? 1 : share < kMostTokens ? share : kMostTokens);
    if (A.tokens > room) A.tokens = (int)room;
    A.token_blocks = narrow && s.heads == 0 ? 0 : (s.B * s.T + A.tokens - 1) / A.tokens;
    A.pages = (int)((s.T + cache->page_tokens - 2) / cache->page_tokens + 1);
    const int64_t blocks = A.token_blocks + (narrow ? s.B * A.pages * cache->heads * 2 : 0), most = ((int64_t)1 << 32) / kThreads - 1;
    if (blocks > most * 65535) return SIG_ERR_TOO_LARGE;
    // (a launch holds fewer than 2^32 threads along an axis)
    const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)((blocks + most - 1) / most));
    with_type(s.type, [&](auto t) {
        using E = typename decltype(t)::type;
        auto go = [&](auto n) {
            constexpr int N = decltype(n)::value, M = kGroup<E>;
            int64_t units = (s.interleaved ? s.turned / N : s.turned / 2 / N) + (cache->key_dim - s.turned + M - 1) / M;
            if (!narrow && (cache->value_dim + M - 1) / M > units) units = (cache->value_dim + M - 1) / M;
            A.places = 1;
            while (A.places < units && A.places < kThreads) A.places *= 2;
            const hipStream_t st = (hipStream_t)hip_stream;
            if constexpr (N > 1) {      // (neighbours are two at least)
                if (s.interleaved && narrow) sig_cache_append_kernel<E, N, true, true><<<grid, kThreads, 0, st>>>(A);
                else if (s.interleaved) sig_cache_append_kernel<E, N, true, false><<<grid, kThreads, 0, st>>>(A);
                if (s.interleaved) return;
            }
            if (narrow) sig_cache_append_kernel<E, N, false, true><<<grid, kThreads, 0, st>>>(A);
            else sig_cache_append_kernel<E, N, false, false><<<grid, kThreads, 0, st>>>(A);
        };
        // the widest loads that the turned components are a whole number of
        constexpr int MOST = kGroup<E>;
        const int64_t whole = s.interleaved ? s.turned : s.turned / 2;
        if (whole % MOST == 0) go(std::integral_constant<int, MOST>());
        else if (whole % (MOST / 2) == 0) go(std::integral_constant<int, MOST / 2>());
        else if (whole % 2 == 0) go(std::integral_constant<int, 2>());
        else go(std::integral_constant<int, 1>());
    });
    return hipGetLastError() == hipSuccess ? SIG_OK : SIG_ERR_HIP;
}
