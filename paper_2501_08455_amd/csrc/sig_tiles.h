// Matrix products of M x M tiles on gfx950 for softmax attention, and the LDS tiles that feed them.
//
// A product's result tile holds, in lane l of a wavefront, column l % M at the rows row_of(l, i), i < REGS.  A fragment is the wavefront's share of an
// operand of M lines and STEP places of the summed axis: lane l holds line l % M.  The order along a summed axis is free as long as
// both operands agree:
//   rows       neighbouring places: lines = rows of an LDS tile, summed axis = its columns.  The other operand is loaded to match
//              (fragment_of)
//   columns    the places that a result tile's registers hold, so that results are operands as they lie: lines = columns of an LDS
//              tile, summed axis = its rows
//
// 16-bit values: 32 x 32 tiles, since each fragment that is read from LDS then feeds twice the products that 16 x 16 has for it.  LDS
// gives 128 bytes a cycle to four matrix units, and a wavefront with 32 lines asks for just that at the units' full rate.  Float32: 16 x 16, an
// eighth of the rate or less, where the wavefront's own operands take half of the registers.
#ifndef SIG_TILES_H
#define SIG_TILES_H

#include <type_traits>

#include "sig_types.h"

namespace sig {

using f4 = __attribute__((ext_vector_type(4))) float;
using f16v = __attribute__((ext_vector_type(16))) float;

template <typename E, int D>
struct LdsTile;

// What bfloat16 and float16 share
template <typename E_>
struct NarrowTiles {
    using E = E_;
    static constexpr int M = 32, STEP = 16, REGS = 16, PLANES = 1;      // planes: of a value in LDS, side by side
    static constexpr int GROUP = 8;                 // values of a fragment's lane
    template <int D>
    using Tile = LdsTile<E, D>;
    using Frag = __attribute__((ext_vector_type(8))) E;
    using Result = f16v;

    static __device__ constexpr int row_of(int lane, int i) { return i / 4 * 8 + lane / 32 * 4 + i % 4; }
    // of the columns form: place along the summed axis of element e
    static __device__ constexpr int place_of(int lane, int e) { return e / 4 * 8 + lane / 32 * 4 + e % 4; }
    // of the rows form: the first of a lane's neighbouring places
    static __device__ constexpr int first_of(int lane) { return lane / 32 * 8; }

    template <typename Tile>
    static __device__ Frag rows(int lane, const E *tile, int line, int at)
    {
        return *(const Frag *)(tile + (lane % 32 * Tile::PITCH + lane / 32 * 8) + (line * Tile::PITCH + at));
    }
    // The transposing LDS read: 16 lanes name the quarters of four rows of 16 values, and lane i receives value i of each row.
    template <typename Tile>
    static __device__ Frag columns(int lane, const E *tile, int at, int line)
    {
        using s4 = __attribute__((ext_vector_type(4))) short;
        using Read = __attribute__((address_space(3))) s4;
        const int i = lane % 16;
        const E *p = tile + ((lane / 32 * 4 + i / 4) * Tile::PITCH + lane / 16 % 2 * 16 + i % 4 * 4);
        const s4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read *)(p + (at * Tile::PITCH + line)));
        const s4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read *)(p + ((at + 8) * Tile::PITCH + line)));
        return __builtin_bit_cast(Frag, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // fragment number `step` of the columns form out of result tiles
    static __device__ Frag of_results(const Result *tiles, int step)
    {
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (E)tiles[step / 2][step % 2 * 8 + e];
        return f;
    }
};

// ... and in 16 x 16 tiles
template <typename E_>
struct SmallNarrowTiles {
    using E = E_;
    static constexpr int M = 16, STEP = 32, REGS = 4, PLANES = 1;
    static constexpr int GROUP = 8;
    template <int D>
    using Tile = LdsTile<E, D>;
    using Frag = __attribute__((ext_vector_type(8))) E;
    using Result = f4;

    static __device__ constexpr int row_of(int lane, int i) { return lane / 16 * 4 + i; }
    static __device__ constexpr int place_of(int lane, int e) { return e / 4 * 16 + lane / 16 * 4 + e % 4; }
    static __device__ constexpr int first_of(int lane) { return lane / 16 * 8; }

    template <typename Tile>
    static __device__ Frag rows(int lane, const E *tile, int line, int at)
    {
        return *(const Frag *)(tile + (lane % 16 * Tile::PITCH + lane / 16 * 8) + (line * Tile::PITCH + at));
    }
    template <typename Tile>
    static __device__ Frag columns(int lane, const E *tile, int at, int line)
    {
        using s4 = __attribute__((ext_vector_type(4))) short;
        using Read = __attribute__((address_space(3))) s4;
        const int i = lane % 16;
        const E *p = tile + ((lane / 16 * 4 + i / 4) * Tile::PITCH + i % 4 * 4);
        const s4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read *)(p + (at * Tile::PITCH + line)));
        const s4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read *)(p + ((at + 16) * Tile::PITCH + line)));
        return __builtin_bit_cast(Frag, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    static __device__ Frag of_results(const Result *tiles, int step)
    {
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (E)tiles[2 * step + e / 4][e % 4];
        return f;
    }
};

// Tiles<E>, and SmallTiles<E> where a line has more than 128 values, of which fewer then fit the registers
template <typename E>
struct Tiles;
template <typename E>
struct SmallTiles;

template <>
struct Tiles<bf16> : NarrowTiles<bf16> {
    static __device__ Result multiply(Frag left, Frag right, Result sum) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(left, right, sum, 0, 0, 0); }
};

template <>
struct Tiles<f16> : NarrowTiles<f16> {
    static __device__ Result multiply(Frag left, Frag right, Result sum) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(left, right, sum, 0, 0, 0); }
};

template <>
struct SmallTiles<bf16> : SmallNarrowTiles<bf16> {
    static __device__ Result multiply(Frag left, Frag right, Result sum) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(left, right, sum, 0, 0, 0); }
};

template <>
struct SmallTiles<f16> : SmallNarrowTiles<f16> {
    static __device__ Result multiply(Frag left, Frag right, Result sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(left, right, sum, 0, 0, 0); }
};

template <>
struct Tiles<float> {
    using E = float;
    static constexpr int M = 16, STEP = 16, REGS = 4, PLANES = 1;
    static constexpr int GROUP = 4;
    template <int D>
    using Tile = LdsTile<E, D>;
    using Frag = f4;
    using Result = f4;

    static __device__ constexpr int row_of(int lane, int i) { return lane / 16 * 4 + i; }
    static __device__ constexpr int place_of(int lane, int e) { return lane / 16 * 4 + e; }
    static __device__ constexpr int first_of(int lane) { return lane / 16 * 4; }

    template <typename Tile>
    static __device__ Frag rows(int lane, const float *tile, int line, int at)
    {
        return *(const Frag *)(tile + (lane % 16 * Tile::PITCH + lane / 16 * 4) + (line * Tile::PITCH + at));
    }
    template <typename Tile>
    static __device__ Frag columns(int lane, const float *tile, int at, int line)
    {
        const float *p = tile + (lane / 16 * 4 * Tile::PITCH + lane % 16) + (at * Tile::PITCH + line);
        return f4{p[0], p[Tile::PITCH], p[2 * Tile::PITCH], p[3 * Tile::PITCH]};
    }
    static __device__ Frag of_results(const Result *tiles, int step) { return tiles[step]; }
    static __device__ Result multiply(Frag left, Frag right, Result sum)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(left[i], right[i], sum, 0, 0, 0);
        return sum;
    }
};

template <>
struct SmallTiles<float> : Tiles<float> {};

// Float32 as three bfloat16 numbers that add up to it, 24 digits in all, multiplied in 32 x 32 tiles: six of the nine products of parts, the others being
// 2^-23 of a product at most and 2^-26 on average, with either sign.  That is 2.7 times the rate that float32 products have, with twice the lines for each read.
// The first part is cut off rather than rounded (so that it does not overflow), the second is rounded, the third is what is left.
struct SplitTiles : NarrowTiles<bf16> {
    using Base = NarrowTiles<bf16>;
    static constexpr int PLANES = 3;
    struct Frag {
        Base::Frag part[PLANES];
    };
    template <int D>
    using Tile = LdsTile<bf16, PLANES * D>;

    // FINITE: x is known not to be infinite (an infinity is its first part).  NANS: a NaN's first part is NaN, whatever its bits (else one that has none in its upper half reads as
    // infinity there, and is NaN by its second part)
    template <bool FINITE, bool NANS, int N, typename V>
    static __device__ void split(const float *given, V *parts)
    {
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = NANS ? __builtin_canonicalizef(given[e]) : given[e];
        using b2 = __attribute__((ext_vector_type(2))) bf16;
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const unsigned low = __builtin_bit_cast(unsigned, x[e]), high = __builtin_bit_cast(unsigned, x[e + 1]);
            float a = x[e] - __builtin_bit_cast(float, low & 0xffff0000u), b = x[e + 1] - __builtin_bit_cast(float, high & 0xffff0000u);
            if (!FINITE) {
                a = fabsf(x[e]) == INFINITY ? 0.0f : a;
                b = fabsf(x[e + 1]) == INFINITY ? 0.0f : b;
            }
            const b2 first = __builtin_bit_cast(b2, __builtin_amdgcn_perm(high, low, 0x07060302u));
            unsigned bits = __builtin_bit_cast(unsigned, b2{(bf16)a, (bf16)b});
            asm("" : "+v"(bits));      // (or the conversion is done anew for each half)
            const b2 second = __builtin_bit_cast(b2, bits);
            a -= __builtin_bit_cast(float, bits << 16);
            b -= __builtin_bit_cast(float, bits & 0xffff0000u);
            const b2 third = __builtin_bit_cast(b2, __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                parts[0][e + i] = first[i];
                parts[1][e + i] = second[i];
                parts[2][e + i] = third[i];
            }
        }
    }
    template <typename Tile>
    static __device__ Frag rows(int lane, const bf16 *tile, int line, int at)
    {
        Frag f;
#pragma unroll
        for (int i = 0; i < PLANES; ++i) f.part[i] = Base::rows<Tile>(lane, tile, line, at + i * (Tile::WIDTH / PLANES));
        return f;
    }
    template <typename Tile>
    static __device__ Frag columns(int lane, const bf16 *tile, int at, int line)
    {
        Frag f;
#pragma unroll
        for (int i = 0; i < PLANES; ++i) f.part[i] = Base::columns<Tile>(lane, tile, at, line + i * (Tile::WIDTH / PLANES));
        return f;
    }
    static __device__ Frag of_results(const Result *tiles, int step)
    {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = tiles[step / 2][step % 2 * 8 + e];
        Frag f;
        split<true, false, 8>(x, f.part);
        return f;
    }
    static __device__ Result multiply(const Frag &left, const Frag &right, Result sum)
    {
#pragma unroll
        for (int both = PLANES - 1; both >= 0; --both)      // (the smallest first)
#pragma unroll
            for (int i = 0; i <= both; ++i) sum = multiply_parts(left, i, right, both - i, sum);
        return sum;
    }
    static __device__ Result multiply_parts(const Frag &left, int i, const Frag &right, int j, Result sum)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(left.part[i], right.part[j], sum, 0, 0, 0);
    }
};

// Fragments as numbers: value e, and setting it
template <typename F>
__device__ inline float fragment_value(const F &f, int e) { return (float)f[e]; }
__device__ inline float fragment_value(const SplitTiles::Frag &f, int e) { return (float)f.part[0][e] + ((float)f.part[1][e] + (float)f.part[2][e]); }
template <typename F, typename V>
__device__ inline void set_fragment(F &f, const V &values)
{
#pragma unroll
    for (int e = 0; e < (int)(sizeof(F) / sizeof(f[0])); ++e) f[e] = (std::remove_reference_t<decltype(f[0])>)values[e];
}
template <typename V>
__device__ inline void set_fragment(SplitTiles::Frag &f, const V &values)
{
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = values[e];
    SplitTiles::split<false, true, 8>(x, f.part);
}

// Rows of D values in LDS, PITCH apart: an odd number of 16 bytes, so that the 16 rows of a 16-byte read (rows) find all 64 banks, and
// one that keeps the 32-byte pieces of four rows of a transposing read in different ones.
template <typename E, int D>
struct LdsTile {
    static constexpr int WIDTH = D, BANK_GROUPS = D * (int)sizeof(E) / 16 % 16;
    static constexpr int PITCH = D + (sizeof(E) == 4 ? 4 : BANK_GROUPS == 0 || BANK_GROUPS == 4 ? 24 : 8);
};

// The wavefront's own operand, one line a lane: a fragment to match step number j of the rows form, zeros where `there` is false
template <typename X, typename T>
__device__ inline void fragment_of(typename X::Frag *f, int lane, int j, const T *line, int dim, bool there, bool negated = false)
{
    constexpr int N = X::GROUP, LOAD = 16 / (int)sizeof(T);
    const int at = j * X::STEP + X::first_of(lane);
    __attribute__((ext_vector_type(N))) T got = {};
    if (there && at + N <= dim) {
#pragma unroll
        for (int first = 0; first < N; first += LOAD) {
            const auto some = __builtin_bit_cast(__attribute__((ext_vector_type(LOAD))) T, load_words<T, LOAD>(line + at + first));
#pragma unroll
            for (int e = 0; e < LOAD; ++e) got[first + e] = some[e];
        }
    } else if (there) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at + e < dim) got[e] = line[at + e];
    }
    if (negated) got = -got;
    set_fragment(*f, got);
}

template <typename X, int STEPS, typename T>
__device__ inline void fragments_of(typename X::Frag *f, int lane, const T *line, int dim, bool there, bool negated)
{
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        fragment_of<X>(f + j, lane, j, line, dim, there, negated);
    }
}

// ROWS x D values, global memory -> registers -> LDS, by THREADS threads: zeros beyond the rows and values that are there.  Loads of whole groups are
// unconditional (what is not there is read from a place that is, and dropped on the way to LDS), so that all are in flight at once.
// WHOLE: rows have D values.  ANEW: addresses are worked out anew each time, where keeping them asks for more registers than there are.
template <typename T, typename X, int D, int ROWS, int THREADS, bool WHOLE, bool ANEW = false>
struct TileMover {
    using E = typename X::E;
    static constexpr int GROUP = 16 / (int)sizeof(T), GROUPS = D / GROUP, COUNT = (ROWS * GROUPS + THREADS - 1) / THREADS;
    static constexpr bool EVEN = ROWS * GROUPS % THREADS == 0;      // else some threads have no last group (they load what is there, and drop it)
    Words<T, GROUP> held[COUNT];

    static __device__ int thread()
    {
        int number = threadIdx.x;
        if (ANEW) asm volatile("" : "+v"(number));
        return number;
    }
    static __device__ int row_of(int i) { return (thread() + i * THREADS) / GROUPS; }
    static __device__ int place_of(int i) { return (thread() + i * THREADS) % GROUPS * GROUP; }

    static __device__ bool here(int i) { return EVEN || (int)threadIdx.x + i * THREADS < ROWS * GROUPS; }

    // rows 0 ... n - 1 are there, n >= 1
    __device__ void load(const T *first, int64_t stride, int dim, int n)
    {
        if (WHOLE || dim >= GROUP) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int place = place_of(i);
                held[i] = load_words<T, GROUP>(first + min(row_of(i), n - 1) * stride + (WHOLE || place + GROUP <= dim ? place : 0));
            }
        }
        if (!WHOLE && dim % GROUP) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int place = place_of(i);
                if (place < dim && place + GROUP > dim) {
                    const T *p = first + min(row_of(i), n - 1) * stride;
                    struct { T v[GROUP]; } rest;
#pragma unroll
                    for (int j = 0; j < GROUP; ++j) {
                        rest.v[j] = (T)0.0f;
                        if (place + j < dim) rest.v[j] = p[place + j];
                    }
                    held[i] = __builtin_bit_cast(Words<T, GROUP>, rest);
                }
            }
        }
    }
    // whether this thread holds something that is not finite
    __device__ bool spoilt(int dim, int n) const
    {
        bool any = false;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            bool bad = false;
#pragma unroll
            for (int j = 0; j < (int)sizeof(held[i]) / 4; ++j) bad |= word_spoilt<T>(held[i][j]);
            const bool there = row_of(i) < n, within = WHOLE || place_of(i) < dim;
            any |= bad & there & within & here(i);
        }
        return any;
    }
    // NANS: see SplitTiles
    template <bool NANS = false>
    __device__ void store(E *tile, int dim, int n) const
    {
        using Tile = typename X::template Tile<D>;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const bool there = row_of(i) < n, within = WHOLE || place_of(i) < dim, ok = there & within;
            E *to = tile + row_of(i) * Tile::PITCH + place_of(i);
            const f4 bits = ok ? __builtin_bit_cast(f4, held[i]) : f4{};
            if constexpr (X::PLANES == 1) {
                if (EVEN || here(i)) *(f4 *)to = bits;
            } else {
                using b4 = __attribute__((ext_vector_type(4))) bf16;
                const float x[] = {bits[0], bits[1], bits[2], bits[3]};
                b4 parts[X::PLANES];
                X::template split<false, NANS, 4>(x, parts);
#pragma unroll
                for (int p = 0; p < X::PLANES; ++p)
                    if (EVEN || here(i)) *(b4 *)(to + p * D) = parts[p];
            }
        }
    }
};

// acc[t] += columns(tile)' x p, tile by tile of D / M: `p` are STEPS fragments along the tile's rows.  Unless WHOLE, only `dim` of the D columns are there,
// and quarters of D that have none are left out.  Between APART steps nothing is moved: else all reads are moved to the front, and more registers
// are asked for than there are.
template <typename X, int D, int STEPS, bool WHOLE, int APART = 1>
__device__ inline void product_along_rows(int lane, const typename X::E *tile, const typename X::Frag *p, typename X::Result *acc, int dim)
{
    constexpr int PIECES = WHOLE ? 1 : 4, TILES = D / X::M / PIECES > 0 ? D / X::M / PIECES : 1;
#pragma unroll
    for (int piece = 0; piece < D / X::M; piece += TILES) {
        if (!WHOLE && piece * X::M >= dim) break;
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
#pragma unroll
            for (int t = piece; t < piece + TILES; ++t) acc[t] = X::multiply(X::template columns<typename X::template Tile<D>>(lane, tile, j * X::STEP, t * X::M), p[j], acc[t]);
            if (j % APART == APART - 1) __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Tiles that are partly hidden and hold something that is not finite: that is set to 0 in LDS before the product along the rows, by all threads ...
template <typename X, int D, int ROWS, int THREADS>
__device__ inline void leave_finite(typename X::E *tile)
{
    using E = typename X::E;
    constexpr int WIDTH = D * X::PLANES;
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < ROWS * WIDTH; i += THREADS) {
        E *x = tile + i / WIDTH * X::template Tile<D>::PITCH + i % WIDTH;
        if (!__builtin_isfinite((float)*x)) *x = (E)0.0f;
    }
    __syncthreads();
}

// ... and behind it added by the lanes whose column sees its row, of the n rows at `first`.  A product counts them: the tile becomes 1 where there is
// one, and the other operand where it is seen.  NANS: as NaN, which is what it comes to where its factors are signed; else NaN, infinity
// and minus infinity as they are, their factors being positive.  By all threads; `idle` wavefronts only help with the tile.
template <typename X, int D, int ROWS, int THREADS, bool NANS, typename T, typename Seen>
__device__ inline void add_not_finite(int lane, typename X::E *tile, const T *first, int64_t stride, int dim, int n, bool idle, typename X::Result *acc, Seen seen)
{
    using E = typename X::E;
#pragma unroll 1
    for (int kind = 0; kind < (NANS ? 1 : 3); ++kind) {
        __syncthreads();
#pragma unroll 1
        for (int i = threadIdx.x; i < ROWS * D; i += THREADS) {
            const int row = i / D, c = i % D;
            const float x = row < n && c < dim ? (float)first[row * stride + c] : 0.0f;
            const bool is = NANS ? !__builtin_isfinite(x) : kind == 0 ? x != x : kind == 1 ? x == INFINITY : x == -INFINITY;
#pragma unroll
            for (int p = 0; p < X::PLANES; ++p) tile[row * X::template Tile<D>::PITCH + c + p * D] = (E)(is && p == 0 ? 1.0f : 0.0f);
        }
        __syncthreads();
        if (idle) continue;
        const float what = kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
        for (int t = 0; t < D / X::M; ++t) {
            typename X::Result counts = {};
#pragma unroll 1
            for (int j = 0; j < ROWS; j += X::STEP) {
                float visible[X::GROUP];
#pragma unroll
                for (int e = 0; e < X::GROUP; ++e) visible[e] = seen(j + X::place_of(lane, e)) ? 1.0f : 0.0f;
                typename X::Frag sees;
                set_fragment(sees, visible);
                counts = X::multiply(X::template columns<typename X::template Tile<D>>(lane, tile, j, t * X::M), sees, counts);
            }
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) acc[t][i] += counts[i] > 0.0f ? what : 0.0f;
        }
    }
}

// s[t] += rows(tile) x own, tile by tile of COUNT M rows (WHOLE, dim, APART: as above)
template <typename X, int D, int COUNT, bool WHOLE, int APART = X::PLANES == 1 ? 2 : 1>
__device__ inline void product_of_rows(int lane, const typename X::E *tile, const typename X::Frag *own, typename X::Result *s, int dim)
{
    constexpr int PIECES = WHOLE ? 1 : 4, STEPS = D / X::STEP / PIECES > 0 ? D / X::STEP / PIECES : 1;
#pragma unroll
    for (int piece = 0; piece < D / X::STEP; piece += STEPS) {
        if (!WHOLE && piece * X::STEP >= dim) break;
#pragma unroll
        for (int step = piece; step < piece + STEPS; ++step) {
#pragma unroll
            for (int t = 0; t < COUNT; ++t) s[t] = X::multiply(X::template rows<typename X::template Tile<D>>(lane, tile, t * X::M, step * X::STEP), own[step], s[t]);
            if (step % APART == APART - 1) __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// An infinity times parts of either sign is no number: where the product of the first parts alone is not finite, that is what the whole product is
template <typename X, int D, int COUNT>
__device__ inline void settle_infinities(int lane, const typename X::E *tile, const typename X::Frag *own, typename X::Result *s)
{
    if constexpr (X::PLANES > 1) {
#pragma unroll
        for (int t = 0; t < COUNT; ++t) {
            typename X::Result first = {};
#pragma unroll
            for (int step = 0; step < D / X::STEP; ++step) {
                first = X::multiply_parts(X::template rows<typename X::template Tile<D>>(lane, tile, t * X::M, step * X::STEP), 0, own[step], 0, first);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < X::REGS; ++i) s[t][i] = __builtin_isfinite(first[i]) ? s[t][i] : first[i];
        }
    }
}

// whether a lane of the wavefront holds something that is not finite
template <int STEPS>
__device__ inline bool any_infinite(const SplitTiles::Frag *f)
{
    bool bad = false;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        const auto words = __builtin_bit_cast(Words<bf16, 8>, f[j].part[0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= word_spoilt<bf16>(words[i]);
    }
    return __any(bad);
}

// The base that probabilities are worked out over, 2^(z - base), for a largest score m: float16's are lifted by 2^LIFT, since what that type holds is small.  (Beyond 2^20 m has no
// digits left for that: a score less its rounded maximum is anything up to 2^-24 of it.)
template <typename E, int LIFT>
__device__ inline float lifted_base(float m)
{
    return std::is_same_v<E, f16> && fabsf(m) < 0x1p20f ? m - LIFT : m;
}

// over the lanes that hold one column of a result tile
template <int M, typename F>
__device__ inline float over_column(float x, F f)
{
    if (M == 16) x = f(x, __shfl_xor(x, 16));
    return f(x, __shfl_xor(x, 32));
}

}  // namespace sig
#endif
