// Matrix products of 16 x 16 tiles on gfx950, for operands kept in bfloat16 or in float32.
//
// A fragment is one wavefront's share of a 16 x STEP operand: lane l (`lane` below, of 64) holds line l % 16 (a row of the left operand, a column of the
// right one; both have the same layout) at 4 SUB places of the summed axis.  A product's result tile holds, in lane l, column
// l % 16 at rows 4 (l / 16) + 0..3.  The order along a summed axis is free as long as both operands agree, so SUB result tiles are
// a fragment as they lie (lines = columns, summed axis = rows), without a detour through LDS, where the other operand is read to match:
//   along_rows     4 SUB neighbouring places, 4 SUB (l / 16) + 0 .. : tile `sub` of a step then has its row r at place(sub, r)
//   along_columns  places 16 sub + 4 (l / 16) + 0..3: tile `sub` has its row r at place 16 sub + r
#ifndef SIG_MATRIX_H
#define SIG_MATRIX_H

#include "sig_types.h"

namespace sig {

using f4 = __attribute__((ext_vector_type(4))) float;
using b4 = __attribute__((ext_vector_type(4))) bf16;
using b8 = __attribute__((ext_vector_type(8))) bf16;
using s4 = __attribute__((ext_vector_type(4))) short;

template <typename E>
struct Matrix;

template <>
struct Matrix<float> {
    using Frag = f4;
    static constexpr int STEP = 16, SUB = 1;
    static constexpr int PAD = 4, COLUMN_PAD = 4;      // values behind a row in LDS that keep the lanes of along_rows, of along_columns in different banks
    static constexpr int EXACT = 1;      // fragments that hold a float32 number whole
    static constexpr int PRODUCTS = 4, COLUMN_READS = 2;      // instructions of multiply() and along_columns()

    static __device__ constexpr int place(int, int r) { return r; }
    // lines = rows of `m` (pitch in values) from `line` on, summed axis = its columns from `at` on
    static __device__ Frag along_rows(int lane, const float *m, int pitch, int line, int at)
    {
        return *(const f4 *)(m + (line + lane % 16) * pitch + at + 4 * (lane / 16));
    }
    // lines = columns of `m`, summed axis = its rows from `at` on.  The columns are those from `line` on, or with GAP the places of tile
    // `sub` of a step that begins there
    template <bool GAP>
    static __device__ Frag along_columns(int lane, const float *m, int pitch, int at, int line, int = 0)
    {
        const float *p = m + (at + 4 * (lane / 16)) * pitch + line + lane % 16;
        return f4{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
    }
    // left x right on top of `sum`
    static __device__ f4 multiply(Frag left, Frag right, f4 sum)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(left[i], right[i], sum, 0, 0, 0);
        return sum;
    }
    // value e of a fragment
    static __device__ float value(Frag f, int e) { return f[e]; }
    // the numbers x[0 .. 3] as PARTS fragments that add up to them
    template <int PARTS>
    static __device__ void split(const float *x, Frag *parts)
    {
        parts[0] = f4{x[0], x[1], x[2], x[3]};
    }
    // the lane's four places of a result tile into the fragments at `to` (PARTS of them, 64 apart), group `sub`
    template <int PARTS>
    static __device__ void put(const float *x, Frag *to, int)
    {
        *to = f4{x[0], x[1], x[2], x[3]};
    }
};

template <>
struct Matrix<bf16> {
    using Frag = b8;
    static constexpr int STEP = 32, SUB = 2;
    static constexpr int PAD = 8, COLUMN_PAD = 16;
    static constexpr int EXACT = 3;      // 3 x 8 digits
    static constexpr int PRODUCTS = 1, COLUMN_READS = 2;

    static __device__ constexpr int place(int sub, int r) { return r / 4 * 8 + 4 * sub + r % 4; }
    static __device__ Frag along_rows(int lane, const bf16 *m, int pitch, int line, int at)
    {
        return *(const b8 *)(m + (line + lane % 16) * pitch + at + 8 * (lane / 16));
    }
    // The transposing LDS read: 16 lanes name the quarters of four rows of 16 values, and lane i receives value i of each row.
    template <bool GAP>
    static __device__ Frag along_columns(int lane, const bf16 *m, int pitch, int at, int line, int sub = 0)
    {
        const int i = lane % 16;
        const bf16 *p = m + (at + 4 * (lane / 16) + i / 4) * pitch + line + 4 * sub + (GAP ? 8 : 4) * (i % 4);
        using Read = __attribute__((address_space(3))) s4;
        const s4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read *)p);
        const s4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read *)(p + 16 * pitch));
        return __builtin_shufflevector(__builtin_bit_cast(b4, low), __builtin_bit_cast(b4, high), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ f4 multiply(Frag left, Frag right, f4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(left, right, sum, 0, 0, 0); }
    static __device__ float value(Frag f, int e) { return (float)f[e]; }
    // x[0 .. 7]; each part holds the next eight digits of what the parts before it leave
    template <int PARTS>
    static __device__ void split(const float *x, Frag *parts)
    {
        digits<PARTS, 8>(x, parts);
    }
    template <int PARTS>
    static __device__ void put(const float *x, Frag *to, int sub)
    {
        b4 parts[PARTS];
        digits<PARTS, 4>(x, parts);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) *((b4 *)(to + 64 * p) + sub) = parts[p];
    }

private:
    // (two at a time, as the conversion takes them; a bfloat16 is the upper half of its float32)
    template <int PARTS, int N, typename V>
    static __device__ void digits(const float *x, V *parts)
    {
        using b2 = __attribute__((ext_vector_type(2))) bf16;
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            float low = x[e], high = x[e + 1];
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                unsigned bits = __builtin_bit_cast(unsigned, b2{(bf16)low, (bf16)high});
                asm("" : "+v"(bits));      // (or the conversion is done anew for each half)
                const b2 pair = __builtin_bit_cast(b2, bits);
                parts[p][e] = pair[0];
                parts[p][e + 1] = pair[1];
                if (p + 1 == PARTS) break;
                low -= __builtin_bit_cast(float, bits << 16);
                high -= __builtin_bit_cast(float, bits & 0xffff0000u);
            }
        }
    }
};

}  // namespace sig
#endif
