// Element types of the sequence operators (enum sig_type) on the device, and the dispatch over them on the host.
#ifndef SIG_TYPES_H
#define SIG_TYPES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sig_sequence.h"

namespace sig {

using bf16 = __bf16;
using f16 = _Float16;

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(bf16 x) { return (float)x; }
__device__ inline float to_float(f16 x) { return (float)x; }

// rounds to nearest, ties to even (what does not fit float16 becomes infinite)
template <typename T>
__device__ inline T from_float(float x) { return (T)x; }

inline bool valid_type(int type) { return type == SIG_F32 || type == SIG_BF16 || type == SIG_F16; }
inline int64_t type_bytes(int type) { return type == SIG_F32 ? 4 : 2; }

template <typename T>
struct Tag {
    using type = T;
};

// f(Tag<element type>) of a valid `type`
template <typename F>
auto with_type(int type, F f)
{
    if (type == SIG_BF16) return f(Tag<bf16>());
    if (type == SIG_F16) return f(Tag<f16>());
    return f(Tag<float>());
}

// N values that are loaded and stored at once; memory is aligned to the element only
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[N];
};

// a pack as the words that it is moved in
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) PackWords {
    __attribute__((ext_vector_type(N * sizeof(T) / 4))) unsigned words;
};

// as one load or store (member by member the compiler may take several)
template <typename T, int N>
__device__ inline Pack<T, N> load_pack(const T *from)
{
    if constexpr (N * sizeof(T) < 4) return *(const Pack<T, N> *)from;
    else return __builtin_bit_cast(Pack<T, N>, ((const PackWords<T, N> *)from)->words);
}

template <typename T, int N>
__device__ inline void store_pack(T *to, const Pack<T, N> &values)
{
    if constexpr (N * sizeof(T) < 4) *(Pack<T, N> *)to = values;
    else ((PackWords<T, N> *)to)->words = __builtin_bit_cast(decltype(PackWords<T, N>::words), values);
}

}  // namespace sig
#endif
