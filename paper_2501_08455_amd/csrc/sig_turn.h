// Angles of rotary positions, for the kernels that turn values.
#ifndef SIG_TURN_H
#define SIG_TURN_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sig_sequence.h"

namespace sig {

// position number `at` of an array of `type` (enum sig_position)
__device__ inline double position_at(const void *positions, int type, int64_t at)
{
    switch (type) {
    case SIG_POSITION_I32: return (double)((const int32_t *)positions)[at];
    case SIG_POSITION_I64: return (double)((const int64_t *)positions)[at];
    case SIG_POSITION_F32: return (double)((const float *)positions)[at];
    default: return ((const double *)positions)[at];
    }
}

// cos and sin of position * frequency.  The turns are reduced in 64 bits: a position of a million times a frequency of one
// radian has no digit left behind the point in 32.
__device__ inline void turn(double position, double frequency, float *c, float *s)
{
    const double turns = position * (frequency * 0.15915494309189535);
    sincospif(2.0f * (float)(turns - rint(turns)), s, c);
}

}  // namespace sig
#endif
