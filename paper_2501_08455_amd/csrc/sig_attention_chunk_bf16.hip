// Linear attention in chunks (sig_attention_chunk.h), bfloat16 operands: products in bfloat16 with float32 sums.
#include "sig_attention_chunk.h"

void sig::launch_chunk_bf16(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st)
{
    launch_chunk<bf16, bf16, 64>(G, nv, output, partial, st);
}
