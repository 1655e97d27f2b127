#include "sig_cache_attention.h"

hipError_t sig::launch_cache_attention_bf16(const CacheAttentionArgs &A, bool narrow, hipStream_t st) { return launch_cache_attention<bf16>(A, narrow, st); }
