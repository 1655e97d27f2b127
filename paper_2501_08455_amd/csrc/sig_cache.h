// The paged cache (include/sig_sequence.h): what the kernels that write to it and read from it share.
#ifndef SIG_CACHE_H
#define SIG_CACHE_H

#include "sig_types.h"

namespace sig {

struct Pages {
    void *values;
    float *scales;              // [pages][heads] of pages of 8 bits
    int64_t page, head, slot;   // strides in values
};

struct CacheArgs {
    Pages keys, values;
    int64_t pages;
    int page_tokens, heads, K, V;
    const int32_t *table;
    int64_t table_pages, table_stride;

    // the page of a place's number `at` along the table of sequence b, or -1
    __device__ int64_t page_of(int64_t b, int64_t at) const
    {
        if (at < 0 || at >= table_pages) return -1;
        const int64_t page = table[b * table_stride + at];
        return page >= 0 && page < pages ? page : -1;
    }
};

using Narrow = uint8_t;      // a value of 8 bits as it is kept: SIG_E4M3
constexpr float kMostNarrow = 448.0f;

__device__ inline float from_narrow(Narrow x) { return __builtin_amdgcn_cvt_f32_fp8(x, 0); }

// rounds to nearest, ties to even; of magnitudes up to 448, what is not finite becomes NaN
__device__ inline Narrow to_narrow(float x)
{
    const int bits = __builtin_amdgcn_cvt_pk_fp8_f32(x, 0.0f, 0, false);
    return __builtin_isfinite(x) ? (Narrow)bits : (Narrow)0x7f;
}

inline bool valid_cache(const sig_cache_t *c, int type)
{
    return c && c->pages >= 0 && c->page_tokens >= 1 && c->heads >= 1 && c->key_dim >= 1 && c->value_dim >= 1 && c->table_pages >= 0 &&
           (c->type == type || c->type == SIG_E4M3) && (c->type != SIG_E4M3 || c->pages == 0 || (c->key_scales && c->value_scales)) &&
           (c->pages == 0 || (c->keys && c->values)) && (c->table_pages == 0 || c->table);
}

inline CacheArgs cache_arguments(const sig_cache_t &c)
{
    return {{c.keys, c.key_scales, c.key_strides[0], c.key_strides[1], c.key_strides[2]},
            {c.values, c.value_scales, c.value_strides[0], c.value_strides[1], c.value_strides[2]},
            c.pages, (int)c.page_tokens, c.heads, c.key_dim, c.value_dim, c.table, c.table_pages, c.table_stride};
}

}  // namespace sig
#endif
