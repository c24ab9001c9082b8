// Angles of position rotations (kda_cache_append.hip, kda_rotate.hip).
#pragma once

#include "kda_common.h"

namespace kda {

// revolutions at a position, less the nearest whole number: exact to 2^-20 of a revolution at 2^31
__device__ __forceinline__ double turns(double frequency, int64_t pos)
{
    const double t = (double)pos * frequency;
    return t - __builtin_rint(t);
}

}  // namespace kda
