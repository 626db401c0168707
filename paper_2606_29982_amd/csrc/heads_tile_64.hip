// Attention with grouped heads of 64 values, many rows.
#include "heads_tile.h"

namespace caee {

hipError_t launch_head_tile_64(const HeadParams& p, unsigned grid, int pieces, hipStream_t s) {
    return head_tile<64>(p, grid, pieces, s);
}

}  // namespace caee
