// Linear attention in chunks (sig_attention_chunk.h), float32 operands: products in float32.
#include "sig_attention_chunk.h"

void sig::launch_chunk_f32(const ChunkArgs &G, int nv, bool output, bool partial, hipStream_t st)
{
    launch_chunk<float, float, 32>(G, nv, output, partial, st);
}
