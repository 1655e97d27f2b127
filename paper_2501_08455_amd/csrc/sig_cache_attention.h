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
constexpr int kMostSplits = 1024;      // (a workgroup's queries times their parts are at most that)

// Float16's probabilities, which are at most 1 here, are lifted by 2^15, and their sum with them (lifted_base).  Down to e^-12 of the largest they then keep the 22 digits
// of their two parts, and below steps of 2^-39 of the largest, instead of 2^-24 (one score 12, 15 and 18 above 1,999 others, whose values are all that counts: the output
// is off by 2.1e-4, its own rounding, instead of 1.1e-3, 2.2e-2 and 0.5; 48 sequences of up to 4,000 places, 16 queries, 32 heads (8 shared) of 128: 252 us both ways).
constexpr int kCacheLift = 15;

// 0 ... 2^31 - 1 over a divisor, as a product
struct Quotient {
    uint64_t factor;
    int shift;
    explicit Quotient(int64_t divisor)
    {
        int bits = 0;
        while (((int64_t)1 << bits) < divisor) ++bits;
        shift = 31 + bits;
        factor = (((uint64_t)1 << shift) + divisor - 1) / divisor;
    }
    Quotient() = default;
    __device__ int operator()(int x) const { return (int)((uint64_t)x * factor >> shift); }
};

struct CacheAttentionArgs {
    CacheArgs cache;
    Quotient quotient;                  // by the tokens of a page
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

// 16 bytes of a row of `dim` values, from value `at` on, as they are kept: row_load, and row_values of what it got when that is used.  The last values of a
// row that is no whole number of loads are the upper ones of a load that ends with the row; beyond the row there are zeros.
using Row = __attribute__((ext_vector_type(4))) unsigned;

template <typename C, bool WHOLE>
__device__ inline Row row_load(const C *row, int at, int dim)
{
    constexpr int COUNT = 16 / sizeof(C), BITS = 8 * sizeof(C);
    if (WHOLE || dim >= COUNT) return load_words<C, COUNT>(row + (WHOLE || at + COUNT <= dim ? at : dim - COUNT));
    using Word = std::conditional_t<sizeof(C) == 1, uint8_t, std::conditional_t<sizeof(C) == 2, uint16_t, uint32_t>>;
    unsigned __int128 bits = 0;
#pragma unroll 1
    for (int j = 0; j < dim; ++j) bits = bits >> BITS | (unsigned __int128)__builtin_bit_cast(Word, row[j]) << (128 - BITS);
    return __builtin_bit_cast(Row, bits);
}
template <typename C, bool WHOLE>
__device__ inline Row row_values(Row got, int at, int dim)
{
    constexpr int COUNT = 16 / sizeof(C), BITS = 8 * sizeof(C);
    if constexpr (WHOLE) return got;
    asm volatile("" : "+s"(dim));      // (compared anew: the answers would be kept in registers)
    const int over = at + COUNT - dim;
    if (dim % COUNT && over > 0 && over < COUNT) got = __builtin_bit_cast(Row, __builtin_bit_cast(unsigned __int128, got) >> (over * BITS));
    return over >= COUNT ? Row{} : got;
}

// values FIRST ... of a row's 16 bytes as an operand's
template <typename X, typename C, int FIRST>
__device__ inline typename X::Frag operand(Row got)
{
    if constexpr (std::is_same_v<C, Narrow>) {
        using Pair = __attribute__((ext_vector_type(2))) bf16;
        Row words;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int word = (int)got[FIRST / 4 + j];
            words[2 * j] = __builtin_bit_cast(unsigned, (Pair)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, 1.0f, false));
            words[2 * j + 1] = __builtin_bit_cast(unsigned, (Pair)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, 1.0f, true));
        }
        return __builtin_bit_cast(typename X::Frag, words);
    } else {
        return __builtin_bit_cast(typename X::Frag, got);
    }
}

constexpr int cache_block(int bytes, int least)
{
    int block = 64;
    while (block > least && block * bytes > 8192) block /= 2;
    return block;
}

// Whether the registers of two workgroups a unit fit (one: 32 x 8,192 places, 8 heads of 192 in 8 bits, queries of bfloat16 184 instead of 153 us; 16 ragged sequences of 8,000,
// 8 heads of 100 float32 208 instead of 147)
template <typename T, typename C, int D, bool WHOLE>
constexpr bool kCachePairs = D <= 128 || (D == 192 && std::is_same_v<C, Narrow> && (WHOLE || sizeof(T) == 2));

// T: of q and out; C: of the cache in memory (Narrow: 8 bits); X: of the products; PARTS: of X's type that hold one of q's or a probability; WHOLE: keys
// and values have D components
template <typename T, typename C, typename X, int D, int QUERY_PARTS, int PARTS, bool WHOLE>
__global__ __launch_bounds__(kCacheThreads, (kCachePairs<T, C, D, WHOLE>) ? 2 : 1) void sig_cache_attention_kernel(CacheAttentionArgs A)
{
    using E = typename X::E;
    using Tile = LdsTile<E, D>;
    constexpr bool NARROW = std::is_same_v<C, Narrow>;
    constexpr int M = X::M, STEPS = D / X::STEP, OUT = D / M, GROUP = X::GROUP;
    // places of a block, 16 to 64: 8 KB of keys as the products want them, or the fewest that a product takes where those are more (so that 64 registers of loads are on their way, 128 at most),
    // and as many of values
    constexpr int BLOCK = cache_block(D * (int)sizeof(E), X::STEP), KEYS = BLOCK / M, PRODUCTS = BLOCK / X::STEP;
    constexpr int LOAD = 16 / (int)sizeof(C), OPERANDS = LOAD / GROUP, KEY_LOADS = STEPS / OPERANDS;      // values of a load, operands that they make
    constexpr int ROW_LOADS = D / LOAD, VALUE_LOADS = BLOCK * ROW_LOADS / 64;
    static_assert(M == kQueries && X::REGS == 4 && BLOCK * ROW_LOADS % 64 == 0 && STEPS % OPERANDS == 0);
    constexpr int ROOM = BLOCK * Tile::PITCH * (int)sizeof(E) > kQueries * D * 4 ? BLOCK * Tile::PITCH * (int)sizeof(E) : kQueries * D * 4;      // bytes
    __shared__ __attribute__((aligned(16))) char room[kCacheWaves][ROOM];
    __shared__ float maxima[kCacheWaves][kQueries], sums[kCacheWaves][kQueries];
    QueryPlace p;
    if (!query_place(A, (int64_t)blockIdx.y * gridDim.x + blockIdx.x, p)) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, K = A.cache.K, V = A.cache.V, column = lane % M;
    E *values = (E *)room[wave];

    // the lane's query, and the places that it sees: those of the window, and the first tokens
    const int64_t number = (int64_t)p.tile * kQueries + column, token = number / A.group;
    const bool there = number < p.count;
    const int own = there ? (int)(p.first + token) : -1;
    const int window = (int)(A.window == 0 || A.window > INT32_MAX ? INT32_MAX : A.window), sinks = (int)(A.sinks > INT32_MAX ? INT32_MAX : A.sinks);
    // (all of it compared, here and below: branches for single values cost more than the comparisons)
    auto seen = [&](int place) { return (place <= own) & ((own - place < window) | (place < sinks)); };
    // The queries, in parts.  A short call is one chain of loads that wait for one another (lengths, table, keys): the queries' go out between the table's and the keys', and
    // are used when those are on their way, but for rows that are not whole, which would ask for more registers than there are (128 sequences of up to 255 places, 4 heads of 64 float32: 16.4 -> 15.2 us, 48 ragged ones in 8 bits with a window 143 -> 136)
    constexpr int QUERY_COUNT = 16 / (int)sizeof(T), QUERY_LOADS = GROUP / QUERY_COUNT;
    // (where the keys' loads have the components of this step)
    auto query_at = [&](int step, int i) { return step / OPERANDS * 4 * LOAD + lane / 16 * LOAD + step % OPERANDS * GROUP + i * QUERY_COUNT; };
    typename X::Frag q[QUERY_PARTS][STEPS];
    auto take_query = [&](int step, int i, Row row) {
        const auto got = __builtin_bit_cast(__attribute__((ext_vector_type(QUERY_COUNT))) T, row_values<T, WHOLE>(row, query_at(step, i), K));
#pragma unroll
        for (int e = 0; e < QUERY_COUNT; ++e) {
            float x = there ? to_float(got[e]) : 0.0f;
            if (A.negated) x = -x;
#pragma unroll
            for (int part = 0; part < QUERY_PARTS; ++part) {
                q[part][step][i * QUERY_COUNT + e] = (E)x;
                x -= (float)q[part][step][i * QUERY_COUNT + e];
                if (x != x) x = 0.0f;      // (infinity less infinity)
            }
        }
    };
    const T *query_line = (const T *)A.q + p.b * A.qs[0] + (there ? token : 0) * A.qs[1] + (p.shared * A.group + (there ? number % A.group : 0)) * A.qs[2];
    if constexpr (!WHOLE) {
#pragma unroll
        for (int step = 0; step < STEPS; ++step)
#pragma unroll
            for (int i = 0; i < QUERY_LOADS; ++i) take_query(step, i, row_load<T, false>(query_line, query_at(step, i), K));
    }

    // blocks of places that some query of the tile sees
    const int64_t from = (int64_t)p.tile * kQueries, until = min(from + kQueries, p.count);
    int low = 0, high = 0, front = 0, count = 0;
    int lowest = 0, highest = -1;      // places of the tile's queries
    if (from < until && A.cache.pages > 0) {
        const int64_t exist = A.cache.table_pages * A.cache.page_tokens;
        lowest = (int)(p.first + from / A.group);
        highest = (int)(p.first + (until - 1) / A.group);
        const int last = (int)min((int64_t)highest, exist - 1);
        low = (int)max((int64_t)0, (int64_t)lowest - window + 1);
        front = (min(sinks, min(low, last + 1)) + BLOCK - 1) / BLOCK;
        low = max(low / BLOCK, front);
        high = last < 0 ? 0 : last / BLOCK + 1;
        count = front + max(0, high - low);
    }
    const int first_block = (int)((int64_t)count * p.split / A.splits), last_block = (int)((int64_t)count * (p.split + 1) / A.splits);
    auto at_of = [&](int j) { return (j < front ? j : low + j - front) * BLOCK; };

    // A block's loads: lane l % BLOCK looks up place l, a block ahead; keys go to where the product wants them, values row by row.  In place of what does not
    // exist the block's first place that does is read, and hidden (another sequence's page may hold anything: NaN there would have the block taken carefully, 128 sequences of up to
    // 255 places, 4 heads of 64 float32 44 us instead of 15); a block without any reads what the first page holds, and is left out.
    int entry = -1;                          // of the table
    auto look_up = [&](int j) {
        const int page = A.quotient(at_of(j) + lane % BLOCK);
        entry = page < A.cache.table_pages ? A.cache.table[p.b * A.cache.table_stride + page] : -1;
    };
    Row keys[KEYS][KEY_LOADS], held[VALUE_LOADS];
    float key_scale = 1.0f, value_scale = 1.0f;
    uint64_t existing = 0;
    int64_t key_row = 0, value_row = 0;      // of the lane's place
    auto find = [&](int j) {
        const int place = at_of(j) + lane % BLOCK, slot = place - A.quotient(place) * A.cache.page_tokens;
        const bool exists = entry >= 0 && entry < A.cache.pages && place < p.n;
        existing = __ballot(exists);
        const int stand_in = __builtin_ctzll(existing | (uint64_t)1 << 63), own_page = exists ? entry : 0, own_slot = exists ? slot : 0;
        const int other_page = __builtin_amdgcn_readlane(own_page, stand_in), other_slot = __builtin_amdgcn_readlane(own_slot, stand_in);
        const int64_t page = exists ? own_page : other_page, in_page = exists ? own_slot : other_slot;
        key_row = page * A.cache.keys.page + p.shared * A.cache.keys.head + in_page * A.cache.keys.slot;
        value_row = page * A.cache.values.page + p.shared * A.cache.values.head + in_page * A.cache.values.slot;
        if constexpr (NARROW) {
            key_scale = A.cache.keys.scales[page * A.cache.heads + p.shared];
            value_scale = A.cache.values.scales[page * A.cache.heads + p.shared];
        }
    };
    auto load_keys = [&] {
#pragma unroll
        for (int t = 0; t < KEYS; ++t) {
            const C *row = (const C *)A.cache.keys.values + __shfl(key_row, t * M + column);
#pragma unroll
            for (int i = 0; i < KEY_LOADS; ++i) keys[t][i] = row_load<C, WHOLE>(row, i * 4 * LOAD + lane / 16 * LOAD, K);
            if (!WHOLE) __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto load_values = [&] {
#pragma unroll
        for (int i = 0; i < VALUE_LOADS; ++i) {
            const C *row = (const C *)A.cache.values.values + __shfl(value_row, (lane + i * 64) / ROW_LOADS);
            held[i] = row_load<C, WHOLE>(row, (lane + i * 64) % ROW_LOADS * LOAD, V);
            if (!WHOLE && i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    };

    typename X::Result acc[OUT] = {};
    float m = -INFINITY, sum = 0.0f;
    bool any = false;
    int j = first_block + wave;
    if (j < last_block) {
        look_up(j);
        Row rows[STEPS][QUERY_LOADS];
        if constexpr (WHOLE) {
#pragma unroll
            for (int step = 0; step < STEPS; ++step)
#pragma unroll
                for (int i = 0; i < QUERY_LOADS; ++i) rows[step][i] = row_load<T, true>(query_line, query_at(step, i), K);
        }
        find(j);
        load_keys();
        load_values();
        if (j + kCacheWaves < last_block) look_up(j + kCacheWaves);
        if constexpr (WHOLE) {
#pragma unroll
            for (int step = 0; step < STEPS; ++step)
#pragma unroll
                for (int i = 0; i < QUERY_LOADS; ++i) take_query(step, i, rows[step][i]);
        }
    }
    // Something that is not finite and not seen by all queries: such blocks are left out, and taken by themselves afterwards (CAREFUL; a branch in
    // the middle would cost every block its registers)
    bool left_out = false;
    auto take = [&](int j, auto careful, bool more) {
        constexpr bool CAREFUL = decltype(careful)::value;
        const int at = at_of(j);
        typename X::Result s[KEYS] = {};
#pragma unroll
        for (int i = 0; i < KEY_LOADS; ++i)
#pragma unroll
            for (int t = 0; t < KEYS; ++t) {
                const Row got = row_values<C, WHOLE>(keys[t][i], i * 4 * LOAD + lane / 16 * LOAD, K);
                const typename X::Frag k = operand<X, C, 0>(got);
#pragma unroll
                for (int part = 0; part < QUERY_PARTS; ++part) s[t] = X::multiply(k, q[part][i * OPERANDS], s[t]);
                if constexpr (OPERANDS == 2) {
                    const typename X::Frag more = operand<X, C, GROUP>(got);
#pragma unroll
                    for (int part = 0; part < QUERY_PARTS; ++part) s[t] = X::multiply(more, q[part][i * OPERANDS + 1], s[t]);
                }
                if (!WHOLE) __builtin_amdgcn_sched_barrier(0);      // (else all operands are made first, and more registers asked for than there are)
            }
        // (the next block's loads go out as soon as there is room for them, so that some are always on their way)
        const uint64_t existed = existing;
        const float key_scales = key_scale, value_scales = value_scale;
        if (more) {
            find(j + kCacheWaves);
            load_keys();
        }
        // whether every query sees every place of the block
        constexpr uint64_t ALL = ~(uint64_t)0 >> (64 - BLOCK);
        const uint64_t exist = existed & ALL;
        const bool all = exist == ALL && at + BLOCK - 1 <= lowest && (highest - at < window || at + BLOCK <= sinks);
        bool spoilt = false;
#pragma unroll
        for (int i = 0; i < VALUE_LOADS; ++i) {
            const int source = (lane + i * 64) / ROW_LOADS;
            E *to = values + source * Tile::PITCH + (lane + i * 64) % ROW_LOADS * LOAD;
            const Row got = row_values<C, WHOLE>(held[i], (lane + i * 64) % ROW_LOADS * LOAD, V);
            *(typename X::Frag *)to = operand<X, C, 0>(got);
            if constexpr (OPERANDS == 2) *(typename X::Frag *)(to + GROUP) = operand<X, C, GROUP>(got);
            if (!all) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (8 bits: NaN is all ones but for the sign)
                    if constexpr (NARROW) spoilt |= (((got[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
                    else spoilt |= word_spoilt<C>(got[e]);
                }
            }
        }
        // (the wavefront's own stores before its own reads: the order that LDS keeps)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (more) {
            load_values();
            if (j + 2 * kCacheWaves < last_block) look_up(j + 2 * kCacheWaves);
        }
        const bool not_finite = !all && __any(spoilt);
        if (exist == 0 || not_finite != CAREFUL) {
            left_out |= exist != 0;
            return;
        }
        if constexpr (NARROW) {
#pragma unroll
            for (int t = 0; t < KEYS; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) s[t][i] *= __shfl(key_scales, t * M + X::row_of(lane, i));
        }
        if (!all) {
#pragma unroll
            for (int t = 0; t < KEYS; ++t)
#pragma unroll
                for (int i = 0; i < X::REGS; ++i) {
                    const int row = t * M + X::row_of(lane, i);
                    const bool ok = (exist >> row & 1) & seen(at + row);
                    any |= ok;
                    s[t][i] = ok ? s[t][i] : -INFINITY;
                }
        }
        __builtin_amdgcn_sched_barrier(0);
        float most = -INFINITY;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) most = fmaxf(most, s[t][i]);
        any |= all & there;
        most = over_column<M>(most, fmaxf);
        const float next = fmaxf(m, most * A.power), base = next == -INFINITY ? 0.0f : lifted_base<E, kCacheLift>(next);
        const float shrink = __builtin_amdgcn_exp2f(lifted_base<E, kCacheLift>(m) - base);
        m = next;
        float total = 0.0f;
#pragma unroll
        for (int t = 0; t < KEYS; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], A.power, -base));
                total += s[t][i];
                // (the values' scale goes into the probabilities: one number for a place instead of one for each of its values)
                if constexpr (NARROW) {
                    const float scale = __shfl(value_scales, t * M + X::row_of(lane, i));
                    s[t][i] = s[t][i] == 0.0f ? 0.0f : s[t][i] * scale;      // (the scale of what is hidden may be anything)
                }
            }
        sum = fmaf(sum, shrink, total);
#pragma unroll
        for (int t = 0; t < OUT; ++t)
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) acc[t][i] *= shrink;
        // (16 bits: two parts of 8 or 11 digits each, since here memory is what bounds and a product more costs nothing)
        typename X::Frag probabilities[PARTS][PRODUCTS];
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int step = 0; step < PRODUCTS; ++step) {
                constexpr int TILES = X::STEP / M;
                probabilities[part][step] = X::of_results(s, step);
                if (part + 1 < PARTS)
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
#pragma unroll
                        for (int i = 0; i < X::REGS; ++i) s[step * TILES + t][i] -= (float)probabilities[part][step][t * X::REGS + i];
            }
        if constexpr (CAREFUL) {
            // query by query, with zeros for what that one does not see
#pragma unroll 1
            for (int c = 0; c < M; ++c) {
                const int its_own = __shfl(own, c);
#pragma unroll
                for (int step = 0; step < PRODUCTS; ++step) {
                    unsigned sees = 0;
#pragma unroll
                    for (int e = 0; e < GROUP; ++e) {
                        const int row = step * X::STEP + X::place_of(lane, e), place = at + row;
                        sees |= ((unsigned)(exist >> row) & (unsigned)((place <= its_own) & ((its_own - place < window) | (place < sinks)))) << e;
                    }
#pragma unroll
                    for (int t = 0; t < OUT; ++t) {
                        typename X::Frag v = X::template columns<Tile>(lane, values, step * X::STEP, t * M);
#pragma unroll
                        for (int e = 0; e < GROUP; ++e) v[e] = sees >> e & 1 ? v[e] : (E)0.0f;
                        typename X::Result r = {};
#pragma unroll
                        for (int part = 0; part < PARTS; ++part) r = X::multiply(v, probabilities[part][step], r);
#pragma unroll
                        for (int i = 0; i < X::REGS; ++i) acc[t][i] += column == c ? r[i] : 0.0f;
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        } else {
#pragma unroll
            for (int step = 0; step < PRODUCTS; ++step)
#pragma unroll
                for (int t = 0; t < OUT; ++t) {
                    const typename X::Frag v = X::template columns<Tile>(lane, values, step * X::STEP, t * M);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) acc[t] = X::multiply(v, probabilities[part][step], acc[t]);
                    if (t % 2) __builtin_amdgcn_sched_barrier(0);
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    for (; j < last_block; j += kCacheWaves) take(j, std::false_type(), j + kCacheWaves < last_block);
    if (left_out) {
#pragma unroll 1
        for (j = first_block + wave; j < last_block; j += kCacheWaves) {
            look_up(j);
            find(j);
            load_keys();
            load_values();
            take(j, std::true_type(), false);
        }
    }

    // the four wavefronts' sums.  One that has seen only scores of minus infinity has a sum of 1 with a maximum of minus infinity, one that has seen
    // nothing 0
    sum = over_column<M>(sum, [](float a, float b) { return a + b; });
    any = over_column<M>(any ? 1.0f : 0.0f, fmaxf) > 0.0f;
    m = lifted_base<E, kCacheLift>(m);
    if (!there) m = -INFINITY, sum = 0.0f;
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

// Joins the parts of cut sequences.  `columns` x `turns` threads (powers of two) take a query, or one of its `slices` of columns: N columns and every
// `turns`-th part each.
template <typename T, int N>
__global__ __launch_bounds__(kCacheThreads) void sig_cache_join_kernel(CacheAttentionArgs A, int columns, int turns, int slices)
{
    __shared__ float shares[kMostSplits], numbers[kCacheThreads / 64];
    __shared__ Pack<float, N> joined[kCacheThreads];
    constexpr int AHEAD = 8, OWN = kMostSplits / kCacheThreads;      // loads on their way; parts whose numbers a thread holds, at most
    const int team = columns * turns, of_team = threadIdx.x % team, first = threadIdx.x - of_team, V = A.cache.V, apart = kQueries * (V + 2);
    const int64_t queries = A.T * A.group, all = A.B * A.cache.heads * queries;
    const int64_t piece = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kCacheThreads / team) + threadIdx.x / team, id = piece / slices;
    const bool there = id < all;
    const int64_t number = there ? id % queries : 0, head = there ? id / queries : 0;
    const float *parts = A.parts + ((head * A.tiles + number / kQueries) * A.splits * kQueries + number % kQueries) * (V + 2);
    float *own_shares = shares + threadIdx.x / team * A.splits;
    // f over what the team's threads hold
    auto over_team = [&](float x, auto f) {
        for (int i = 1; i < team && i < 64; i *= 2) x = f(x, __shfl_xor(x, i));
        if (team <= 64) return x;
        __syncthreads();
        if (threadIdx.x % 64 == 0) numbers[threadIdx.x / 64] = x;
        __syncthreads();
        x = numbers[first / 64];
        for (int i = 1; i < team / 64; ++i) x = f(x, numbers[first / 64 + i]);
        return x;
    };
    // all loads at once: the parts' maxima and sums, and the first of their columns
    float tops[OWN], sums[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int s = of_team + i * team;
        tops[i] = s < A.splits ? parts[(int64_t)s * apart + V] : -INFINITY;
        sums[i] = s < A.splits ? parts[(int64_t)s * apart + V + 1] : 0.0f;
    }
    const int turn = of_team / columns;
    const int c = ((int)(piece % slices) * columns + of_team % columns) * N;      // (V <= slices columns N)
    Pack<float, N> ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const int s = turn + i * turns;
        if (c < V && s < A.splits) ahead[i] = load_pack<float, N>(parts + (int64_t)s * apart + c);
    }
    float top = -INFINITY, total = 0.0f, any = 0.0f;
#pragma unroll
    for (int i = 0; i < OWN; ++i) top = fmaxf(top, tops[i]);
    top = over_team(top, fmaxf);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const float share = __builtin_amdgcn_exp2f(tops[i] - base);
        if (sums[i] != 0.0f) any = 1.0f;
        total = fmaf(sums[i], share, total);
        if (of_team + i * team < A.splits) own_shares[of_team + i * team] = sums[i] != 0.0f ? share : -1.0f;      // (a part that has seen nothing is left out)
    }
    total = over_team(total, [](float a, float b) { return a + b; });
    any = over_team(any, fmaxf);
    __syncthreads();
    float value[N] = {};
    auto add = [&](const Pack<float, N> &part, float share) {
#pragma unroll
        for (int j = 0; j < N; ++j) value[j] = share < 0.0f ? value[j] : fmaf(part.v[j], share, value[j]);
    };
    if (c < V) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (turn + i * turns < A.splits) add(ahead[i], own_shares[turn + i * turns]);
#pragma unroll 8
        for (int s = turn + AHEAD * turns; s < A.splits; s += turns) add(load_pack<float, N>(parts + (int64_t)s * apart + c), own_shares[s]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) joined[threadIdx.x].v[j] = value[j];
    __syncthreads();
    if (turn > 0 || !there || c >= V) return;
    for (int i = 1; i < turns; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) value[j] += joined[threadIdx.x + i * columns].v[j];
    Pack<T, N> result;
#pragma unroll
    for (int j = 0; j < N; ++j) result.v[j] = from_float<T>(any != 0.0f ? value[j] / total : 0.0f);
    store_pack((T *)A.out + ((head / A.cache.heads * A.T + number / A.group) * A.heads + head % A.cache.heads * A.group + number % A.group) * V + c, result);
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
        auto launch = [&](auto whole) {
            constexpr bool WHOLE = decltype(whole)::value, WIDE = sizeof(T) == 4;
            // values of 8 bits are bfloat16's, and a query is one, two or three of them
            if constexpr (D % 64 == 0) {
                if (narrow) sig_cache_attention_kernel<T, Narrow, SmallTiles<bf16>, D, WIDE ? 3 : std::is_same_v<T, f16> ? 2 : 1, WIDE ? 3 : 2, WHOLE><<<grid, kCacheThreads, 0, st>>>(A);
            }
            if (!narrow) sig_cache_attention_kernel<T, T, SmallTiles<T>, D, 1, WIDE ? 1 : 2, WHOLE><<<grid, kCacheThreads, 0, st>>>(A);
        };
        if (A.cache.K == D && A.cache.V == D) launch(std::true_type());
        else launch(std::false_type());
    };
    const int dim = A.cache.K > A.cache.V ? A.cache.K : A.cache.V;
    // (rows of up to 32, and of 65 to 96 and 129 to 192 components in instances of their own: 128 x 8,000 places, 4 heads of 32 float32 338 -> 190 us, 32 x 8,192, 8 heads of 80 bfloat16
    // 160 -> 136, 16 ragged sequences of 2,000, 8 heads of 96 float32 72 -> 33, 32 x 8,192, 8 heads of 192 bfloat16 406 -> 280.  A load of 8-bit keys is two operands, which 32 and 96 are no whole number of)
    if (dim <= 32 && !narrow) go(std::integral_constant<int, 32>());
    else if (dim <= 64) go(std::integral_constant<int, 64>());
    else if (dim <= 96 && !narrow) go(std::integral_constant<int, 96>());
    else if (dim <= 128) go(std::integral_constant<int, 128>());
    else if (dim <= 192) go(std::integral_constant<int, 192>());
    else go(std::integral_constant<int, 256>());
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !A.parts) return e;
    const int64_t queries = A.B * A.cache.heads * A.T * A.group;
    auto join = [&](auto n) {
        constexpr int N = decltype(n)::value;
        int columns = 1, turns = 1, slices = 1;
        while (columns * N < A.cache.V) columns *= 2;
        // (many parts of few queries: eight columns a workgroup, 256 parts of 16 queries 20 -> 10 us)
        for (; A.splits >= 64 && columns > 8; columns /= 2) slices *= 2;
        while (turns < A.splits && columns * turns < kCacheThreads) turns *= 2;
        const int at_once = kCacheThreads / (columns * turns);
        sig_cache_join_kernel<T, N><<<cache_grid((queries * slices + at_once - 1) / at_once), kCacheThreads, 0, st>>>(A, columns, turns, slices);
    };
    if (A.cache.V % 4 == 0) join(std::integral_constant<int, 4>());
    else join(std::integral_constant<int, 1>());
    return hipGetLastError();
}

}  // namespace sig
#endif
