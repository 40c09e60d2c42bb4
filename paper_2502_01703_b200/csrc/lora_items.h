// The items of lora_factors_kernel and the order in which its blocks take them. Plain C++ too, so that it can be checked on the host.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define QLESS_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define QLESS_HOST_DEVICE inline
#endif

namespace qless {

struct FactorItem {
    int32_t slice;                          // of the channels
    int64_t tile;                           // of 128 tokens
    bool is_x;                              // codes (H) or dY (U)
};

// Items 2 m and 2 m + 1 are the two kinds of one token tile and slice. Block b of a grid of G takes items b, b + G, b + 2 G, ...; the
// kinds are to alternate on that way, so that at any time half of the blocks read codes (bound by the work per block of codes) and half
// dY (bound by its bytes). Where G is odd the item's own parity alternates; where it is even (2 m and 2 m + 1 then fall in the same round)
// the parity is turned over every round.
QLESS_HOST_DEVICE FactorItem factor_item(int64_t item, int64_t token_tiles, int64_t grid)
{
    FactorItem f;
    f.slice = (int32_t)(item / (2 * token_tiles));
    const int64_t r = item - f.slice * (2 * token_tiles);
    const int64_t round = grid % 2 == 0 ? item / grid : 0;
    f.is_x = ((r + round) & 1) != 0;
    f.tile = r >> 1;
    return f;
}

}  // namespace qless
