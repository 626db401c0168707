// Attention with grouped heads of 64 values, many rows.
#include "heads_tile.h"

namespace caee {

hipError_t launch_head_tile_64(const HeadParams& p, bool split, unsigned grid, int tiles, hipStream_t s) {
    if (p.tree) return split ? head_tile<64, true, true>(p, grid, tiles, s) : head_tile<64, false, true>(p, grid, tiles, s);
    return split ? head_tile<64, true, false>(p, grid, tiles, s) : head_tile<64, false, false>(p, grid, tiles, s);
}

}  // namespace caee
