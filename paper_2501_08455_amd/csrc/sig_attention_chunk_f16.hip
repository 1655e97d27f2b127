// Linear attention in chunks (sig_attention_chunk.h), float16 operands: widened to float32 on their way into LDS, since sums of products of two do not fit float16.
#include "sig_attention_chunk.h"

void sig::launch_chunk_f16(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st)
{
    launch_chunk<f16, float, 32>(G, nv, output, partial, st);
}
