// Attention with grouped heads of 128 values, many rows.
#include "heads_tile.h"

namespace caee {

hipError_t launch_head_tile_128(const HeadParams& p, unsigned grid, int pieces, hipStream_t s) {
    return head_tile<128>(p, grid, pieces, s);
}

}  // namespace caee
