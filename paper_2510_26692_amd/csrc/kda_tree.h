// Draft trees as kernels read them (kda_cache_tree.hip, kda_tree_steps.hip).
#pragma once

#include "kda_common.h"

namespace kda {

constexpr int kTreeTokens = 64;      // the largest tree: a token a lane

// What lane t's token, with the parent `up`, has above it: itself and its ancestors as bits, none where there is no such token.  Every lane of
// the wave takes part.  (Six doublings: after i of them a lane has its next 2^i ancestors, and the number of the one behind them.)
__device__ __forceinline__ uint64_t tree_line(int32_t up, int tokens)
{
    const int lane = threadIdx.x & 63;
    bool there = up >= -1 && up < lane && lane < tokens;
    up = there ? up : -1;
    uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const int from = up < 0 ? lane : up;
        const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
        const int32_t next = __shfl(up, from);
        const bool ok = __shfl((int)there, from);
        if (up >= 0) {
            lo |= l;
            hi |= h;
            there = there && ok;
            up = next;
        }
    }
    return there ? (uint64_t)hi << 32 | lo : 0ull;
}

}  // namespace kda
