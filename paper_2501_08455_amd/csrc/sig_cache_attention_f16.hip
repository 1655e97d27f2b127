#include "sig_cache_attention.h"

hipError_t sig::launch_cache_attention_f16(const CacheAttentionArgs &A, bool narrow, hipStream_t st) { return launch_cache_attention<f16>(A, narrow, st); }
