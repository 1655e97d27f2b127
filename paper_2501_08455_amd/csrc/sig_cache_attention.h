// Softmax attention of a sequence's last tokens over its paged cache: kernels (include/sig_sequence.h; the formulas are those of sig_window.h).
//
// Queries of heads that share keys stand side by side: 16 of them are the columns of all products, token after token, the heads of a token next to each other.
// A wavefront takes blocks of BLOCK places by itself: keys go from memory into registers as the left operand that they are, values through
// its own part of LDS, out of which they are read transposed.  The next block's loads are on their way meanwhile, and no wavefront waits for
// another until the end, when a workgroup's four join their sums.  Few queries are cut along their places, and a second launch joins the parts.
//
// Bound by memory: each visible page is read once for 16 queries.
#ifndef SIG_CACHE_ATTENTION_H
#define SIG_CACHE_ATTENTION_H

#include <cfloat>

#include "sig_cache.h"
#include "sig_internal.h"
#include "sig_tiles.h"

namespace sig {

constexpr int kCacheThreads = 256, kCacheWaves = kCacheThreads / 64;
constexpr int kQueries = 16;      // of a workgroup

struct CacheAttentionArgs {
    CacheArgs cache;
    const void *q;
    int64_t qs[3];
    const int64_t *lengths, *counts;
    void *out;                          // [B][T][heads][V]
    float *parts;                       // [B * shared heads * tiles][splits][16][V + 2], or null where there is one split
    int64_t B, T;
    int heads, group;
    int64_t window, sinks;              // window 0: none
    float power;                        // |scale| log2(e)
    int negated;
    int tiles, splits;                  // of 16 queries; of the places
};

struct QueryPlace {
    int64_t b, n, first;      // sequence; tokens that it holds; place of its query number 0
    int64_t line;             // number of the workgroup's queries among all
    int shared, tile, split;
    int64_t count;            // queries of the sequence, all heads of a shared one
};

__device__ inline bool query_place(const CacheAttentionArgs &A, int64_t id, QueryPlace &p)
{
    p.split = (int)(id % A.splits);
    p.line = id / A.splits;
    p.tile = (int)(p.line % A.tiles);
    const int64_t head = p.line / A.tiles;
    p.shared = (int)(head % A.cache.heads);
    p.b = head / A.cache.heads;
    if (p.b >= A.B) return false;
    const int64_t n = A.lengths[p.b], most = (int64_t)INT32_MAX - 1023, counted = A.counts ? A.counts[p.b] : A.T;
    p.n = n < 0 ? 0 : n > most ? most : n;
    const int64_t count = counted < 0 ? 0 : counted > A.T ? A.T : counted;
    p.first = p.n - count;
    p.count = count * A.group;
    return true;
}

// what is not finite left out, or 1 where there is what `kind` counts: NaN, infinity, minus infinity
template <typename X>
__device__ inline typename X::Frag only_finite(typename X::Frag f)
{
#pragma unroll
    for (int e = 0; e < X::GROUP; ++e) f[e] = __builtin_isfinite((float)f[e]) ? f[e] : (typename X::E)0.0f;
    return f;
}
template <typename X>
__device__ inline typename X::Frag only_kind(typename X::Frag f, int kind)
{
#pragma unroll
    for (int e = 0; e < X::GROUP; ++e) {
        const float x = (float)f[e];
        f[e] = (typename X::E)((kind == 0 ? x != x : kind == 1 ? x == INFINITY : x == -INFINITY) ? 1.0f : 0.0f);
    }
    return f;
}

// GROUP values of a row of `dim` from component `at` on, as they are kept; zeros beyond the row
template <typename C, int GROUP>
__device__ inline Pack<C, GROUP> row_values(const C *row, int at, int dim)
{
    Pack<C, GROUP> got = {};
    if (at + GROUP <= dim) {
        got = load_pack<C, GROUP>(row + at);
    } else {
#pragma unroll
        for (int j = 0; j < GROUP; ++j)
            if (at + j < dim) got.v[j] = row[at + j];
    }
    return got;
}

template <typename E, typename C>
__device__ inline E widened(C x)
{
    if constexpr (std::is_same_v<C, Narrow>) return (E)from_narrow(x);
    else return (E)x;
}

// T: of q and out; C: of the cache in memory (Narrow: 8 bits); X: of the products
template <typename T, typename C, typename X, int D>
__global__ __launch_bounds__(kCacheThreads, D * sizeof(typename X::E) <= 256 ? 2 : 1) void sig_cache_attention_kernel(CacheAttentionArgs A)
{
    using E = typename X::E;
    using Tile = LdsTile<E, D>;
    constexpr bool NARROW = std::is_same_v<C, Narrow>;
    constexpr int M = X::M, BLOCK = X::STEP, KEYS = BLOCK / M, STEPS = D / X::STEP, OUT = D / M, GROUP = X::GROUP, PARTS = sizeof(E) == 2 ? 2 : 1;
    static_assert(M == kQueries && X::REGS == 4);
    constexpr int ROOM = BLOCK * Tile::PITCH * (int)sizeof(E) > kQueries * D * 4 ? BLOCK * Tile::PITCH * (int)sizeof(E) : kQueries * D * 4;      // bytes
    __shared__ __attribute__((aligned(16))) char room[kCacheWaves][ROOM];
    __shared__ float maxima[kCacheWaves][kQueries], sums[kCacheWaves][kQueries];
    QueryPlace p;
    if (!query_place(A, (int64_t)blockIdx.y * gridDim.x + blockIdx.x, p)) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, K = A.cache.K, V = A.cache.V, column = lane % M;
    E *values = (E *)room[wave];

    // the lane's query, and the places that it sees: those of the window from `low` on, and the first tokens
    const int64_t number = (int64_t)p.tile * kQueries + column, token = number / A.group;
    const bool there = number < p.count;
    const int own = there ? (int)(p.first + token) : -1;
    const int window = (int)(A.window == 0 || A.window > INT32_MAX ? INT32_MAX : A.window), sinks = (int)(A.sinks > INT32_MAX ? INT32_MAX : A.sinks);
    auto seen = [&](int place) { return place <= own && (own - place < window || place < sinks); };
    typename X::Frag q[STEPS];
    fragments_of<X, STEPS>(q, lane, (const T *)A.q + p.b * A.qs[0] + (there ? token : 0) * A.qs[1] + (p.shared * A.group + (there ? number % A.group : 0)) * A.qs[2], K, there, A.negated);

    // blocks of places that some query of the tile sees
    const int64_t from = (int64_t)p.tile * kQueries, until = min(from + kQueries, p.count);
    int low = 0, high = 0, front = 0, count = 0;
    if (from < until) {
        const int64_t exist = A.cache.table_pages * A.cache.page_tokens;
        const int highest = (int)min(p.first + (until - 1) / A.group, exist - 1);
        low = (int)max((int64_t)0, p.first + from / A.group - window + 1);
        front = (min(sinks, min(low, highest + 1)) + BLOCK - 1) / BLOCK;
        low = max(low / BLOCK, front);
        high = highest < 0 ? 0 : highest / BLOCK + 1;
        count = front + max(0, high - low);
    }
    const int first_block = (int)((int64_t)count * p.split / A.splits), last_block = (int)((int64_t)count * (p.split + 1) / A.splits);
    auto at_of = [&](int j) { return (j < front ? j : low + j - front) * BLOCK; };

    // a block's loads: lane l % BLOCK looks up place l, keys go to where the product wants them, values row by row
    constexpr int ROW_GROUPS = D / GROUP, LOADS = BLOCK * ROW_GROUPS / 64;
    static_assert(BLOCK * ROW_GROUPS % 64 == 0);
    Pack<C, GROUP> keys[KEYS][STEPS], held[LOADS];
    int64_t key_row = 0, value_row = 0;      // of the lane's place
    float key_scale = 1.0f, value_scale = 1.0f;
    bool exists = false;                     // ... and is seen by some query
    auto load = [&](int j) {
        const int place = at_of(j) + lane % BLOCK;
        const int64_t page = A.cache.page_of(p.b, place / A.cache.page_tokens), slot = place % A.cache.page_tokens;
        // (places that no query sees are not read)
        exists = page >= 0 && place < high * BLOCK && place < p.n;
        const int64_t at = exists ? page : 0;
        key_row = at * A.cache.keys.page + p.shared * A.cache.keys.head + (exists ? slot : 0) * A.cache.keys.slot;
        value_row = at * A.cache.values.page + p.shared * A.cache.values.head + (exists ? slot : 0) * A.cache.values.slot;
        if constexpr (NARROW) {
            key_scale = exists ? A.cache.keys.scales[at * A.cache.heads + p.shared] : 0.0f;
            value_scale = exists ? A.cache.values.scales[at * A.cache.heads + p.shared] : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < KEYS; ++t) {
            const int source = t * M + column;
            const bool ok = __shfl((int)exists, source);
            const C *row = (const C *)A.cache.keys.values + __shfl(key_row, source);
#pragma unroll
            for (int step = 0; step < STEPS; ++step) {
                keys[t][step] = Pack<C, GROUP>{};
                if (ok) keys[t][step] = row_values<C, GROUP>(row, step * X::STEP + X::first_of(lane), K);
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int number = lane + i * 64, source = number / ROW_GROUPS;
            const bool ok = __shfl((int)exists, source);
            const C *row = (const C *)A.cache.values.values + __shfl(value_row, source);
            held[i] = Pack<C, GROUP>{};
            if (ok) held[i] = row_values<C, GROUP>(row, number % ROW_GROUPS * GROUP, V);
        }
    };

    typename X::Result acc[OUT] = {};
    float m = -INFINITY, sum = 0.0f;
    bool any = false;
    int j = first_block + wave;
    if (j < last_block) load(j);
    for (; j < last_block; j += kCacheWaves) {
        const int at = at_of(j);
        typename X::Result s[KEYS] = {};
#pragma unroll
        for (int step = 0; step < STEPS; ++step)
#pragma unroll
            for (int t = 0; t < KEYS; ++t) {
                typename X::Frag k;
#pragma unroll
                for (int e = 0; e < GROUP; ++e) k[e] = widened<E>(keys[t][step].v[e]);
                s[t] = X::multiply(k, q[step], s[t]);
            }
        bool spoilt = false;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int number = lane + i * 64, source = number / ROW_GROUPS;
            const float scale = NARROW ? __shfl(value_scale, source) : 1.0f;
            struct { E v[GROUP]; } row;
#pragma unroll
            for (int e = 0; e < GROUP; ++e) {
                row.v[e] = widened<E>(held[i].v[e]);
                if constexpr (NARROW) row.v[e] = (E)((float)row.v[e] * scale);
                spoilt = spoilt || !__builtin_isfinite((float)row.v[e]);
            }
            *(f4 *)(values + source * Tile::PITCH + number % ROW_GROUPS * GROUP) = __builtin_bit_cast(f4, row);
        }
        spoilt = __any(spoilt);
        const bool existed = exists;
        const float key_scales = key_scale;
        // (the wavefront's own stores before its own reads: the order that LDS keeps)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (j + kCacheWaves < last_block) load(j + kCacheWaves);
        float most = -INFINITY;
        bool hidden = false;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                const int row = t * M + X::row_of(lane, i);
                if constexpr (NARROW) s[t][i] *= __shfl(key_scales, row);
                const bool exists_there = __shfl((int)existed, row), ok = exists_there && seen(at + row);
                any = any || ok;
                hidden = hidden || !ok;
                s[t][i] = ok ? s[t][i] : -INFINITY;
                most = fmaxf(most, s[t][i]);
            }
        most = over_column<M>(most, fmaxf);
        const float next = fmaxf(m, most * A.power), base = next == -INFINITY ? 0.0f : next;
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
        typename X::Frag probabilities[PARTS];
#pragma unroll
        for (int part_of = 0; part_of < PARTS; ++part_of) {
            probabilities[part_of] = X::of_results(s, 0);
            if (part_of + 1 < PARTS)
#pragma unroll
                for (int t = 0; t < KEYS; ++t)
#pragma unroll
                    for (int i = 0; i < X::REGS; ++i) s[t][i] -= (float)probabilities[part_of][t * X::REGS + i];
        }
        if (spoilt && __any(hidden)) {
            // what is not finite counts for the queries that see it (see sig_window.h)
            typename X::Frag sees;
#pragma unroll
            for (int e = 0; e < GROUP; ++e) {
                const bool exists_there = __shfl((int)existed, X::place_of(lane, e));
                sees[e] = (E)(exists_there && seen(at + X::place_of(lane, e)) ? 1.0f : 0.0f);
            }
#pragma unroll
            for (int t = 0; t < OUT; ++t) {
                const typename X::Frag v = X::template columns<Tile>(lane, values, 0, t * M);
#pragma unroll
                for (int part_of = 0; part_of < PARTS; ++part_of) acc[t] = X::multiply(only_finite<X>(v), probabilities[part_of], acc[t]);
#pragma unroll 1
                for (int kind = 0; kind < 3; ++kind) {
                    const typename X::Result counts = X::multiply(only_kind<X>(v, kind), sees, typename X::Result{});
                    const float what = kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
                    for (int i = 0; i < X::REGS; ++i) acc[t][i] += counts[i] > 0.0f ? what : 0.0f;
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < OUT; ++t) {
                const typename X::Frag v = X::template columns<Tile>(lane, values, 0, t * M);
#pragma unroll
                for (int part_of = 0; part_of < PARTS; ++part_of) acc[t] = X::multiply(v, probabilities[part_of], acc[t]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    // the four wavefronts' sums.  One that has seen only scores of minus infinity has a sum of 1 with a maximum of minus infinity, one that has seen
    // nothing 0
    sum = over_column<M>(sum, [](float a, float b) { return a + b; });
    any = over_column<M>(any ? 1.0f : 0.0f, fmaxf) > 0.0f;
    if (m == -INFINITY && sum == sum) sum = any ? 1.0f : 0.0f;
    float *own_sums = (float *)room[wave];
#pragma unroll
    for (int t = 0; t < OUT; ++t) *(f4 *)(own_sums + column * D + t * M + X::row_of(lane, 0)) = acc[t];
    if (lane < M) {
        maxima[wave][lane] = m;
        sums[wave][lane] = sum;
    }
    __syncthreads();
    T *out = (T *)A.out;
    for (int i = threadIdx.x; i < kQueries * (V + 2); i += kCacheThreads) {
        const int query = i / (V + 2), c = i % (V + 2);
        const int64_t number_of = (int64_t)p.tile * kQueries + query;
        if (number_of >= A.T * A.group) continue;
        float top = -INFINITY, total = 0.0f, value = 0.0f;
        bool seen_any = false;
#pragma unroll
        for (int w = 0; w < kCacheWaves; ++w) top = fmaxf(top, maxima[w][query]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int w = 0; w < kCacheWaves; ++w) {
            const float share = __builtin_amdgcn_exp2f(maxima[w][query] - base);
            seen_any = seen_any || sums[w][query] != 0.0f;
            total = fmaf(sums[w][query], share, total);
            if (c < V && sums[w][query] != 0.0f) value = fmaf(((const float *)room[w])[query * D + c], share, value);
        }
        if (A.parts) {
            float *part = A.parts + ((p.line * A.splits + p.split) * kQueries + query) * (V + 2);
            part[c] = c < V ? value : c == V ? top : top == -INFINITY && total == total ? (seen_any ? 1.0f : 0.0f) : total;
        } else if (c < V) {
            const float x = !seen_any ? 0.0f : value / total;
            out[((p.b * A.T + number_of / A.group) * A.heads + p.shared * A.group + number_of % A.group) * V + c] = from_float<T>(x);
        }
    }
}

// Joins the parts of cut sequences: 16 queries a workgroup
template <typename T>
__global__ __launch_bounds__(kCacheThreads) void sig_cache_join_kernel(CacheAttentionArgs A)
{
    QueryPlace p;
    const int64_t line = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (!query_place(A, line * A.splits, p)) return;
    const int V = A.cache.V;
    T *out = (T *)A.out;
    for (int i = threadIdx.x; i < kQueries * V; i += kCacheThreads) {
        const int query = i / V, c = i % V;
        const int64_t number = (int64_t)p.tile * kQueries + query;
        if (number >= A.T * A.group) continue;
        const float *parts = A.parts + (line * A.splits * kQueries + query) * (V + 2);
        const int64_t apart = (int64_t)kQueries * (V + 2);
        float top = -INFINITY, total = 0.0f, value = 0.0f;
        bool any = false;
        for (int s = 0; s < A.splits; ++s) top = fmaxf(top, parts[s * apart + V]);
        const float base = top == -INFINITY ? 0.0f : top;
        for (int s = 0; s < A.splits; ++s) {
            const float sum = parts[s * apart + V + 1], share = __builtin_amdgcn_exp2f(parts[s * apart + V] - base);
            any = any || sum != 0.0f;
            total = fmaf(sum, share, total);
            if (sum != 0.0f) value = fmaf(parts[s * apart + c], share, value);
        }
        out[((p.b * A.T + number / A.group) * A.heads + p.shared * A.group + number % A.group) * V + c] = from_float<T>(any ? value / total : 0.0f);
    }
}

hipError_t launch_cache_attention_f32(const CacheAttentionArgs &A, bool narrow, hipStream_t st);
hipError_t launch_cache_attention_bf16(const CacheAttentionArgs &A, bool narrow, hipStream_t st);
hipError_t launch_cache_attention_f16(const CacheAttentionArgs &A, bool narrow, hipStream_t st);

inline dim3 cache_grid(int64_t blocks)
{
    const int64_t across = ((int64_t)1 << 32) / kCacheThreads - 1;      // (a launch holds fewer than 2^32 threads along an axis)
    return dim3((unsigned)(blocks < across ? blocks : across), (unsigned)((blocks + across - 1) / across));
}

template <typename T>
hipError_t launch_cache_attention(const CacheAttentionArgs &A, bool narrow, hipStream_t st)
{
    const int64_t lines = A.B * A.cache.heads * A.tiles;
    const dim3 grid = cache_grid(lines * A.splits);
    auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (narrow) sig_cache_attention_kernel<T, Narrow, SmallTiles<T>, D><<<grid, kCacheThreads, 0, st>>>(A);
        else sig_cache_attention_kernel<T, T, SmallTiles<T>, D><<<grid, kCacheThreads, 0, st>>>(A);
    };
    const int dim = A.cache.K > A.cache.V ? A.cache.K : A.cache.V;
    if (dim <= 64) go(std::integral_constant<int, 64>());
    else if (dim <= 128) go(std::integral_constant<int, 128>());
    else go(std::integral_constant<int, 256>());
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !A.parts) return e;
    sig_cache_join_kernel<T><<<cache_grid(lines), kCacheThreads, 0, st>>>(A);
    return hipGetLastError();
}

}  // namespace sig
#endif
