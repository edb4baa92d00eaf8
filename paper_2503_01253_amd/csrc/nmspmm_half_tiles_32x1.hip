// The tiled kernel's instantiations for 32-column gathers.
#include "nmspmm_half_launch.h"

namespace nmspmm {

const HalfTileInfo *half_tiles_32x1(int *count)
{
    //                          MI CT NG RT WR WC WK NB LDS
    static const HalfTileInfo list[] = {
        half_tile_info<HalfTile<32, 1, 1, 8, 1, 8, 1, 2, 160>>(),
        half_tile_info<HalfTile<32, 1, 1, 4, 1, 8, 1, 1, 80>>(),
        half_tile_info<HalfTile<32, 1, 1, 4, 1, 4, 2, 1, 80>>(),
        half_tile_info<HalfTile<32, 1, 1, 2, 1, 4, 2, 1, 80>>(),
        half_tile_info<HalfTile<32, 1, 1, 2, 1, 2, 4, 1, 80>>(),
        half_tile_info<HalfTile<32, 1, 1, 1, 1, 2, 4, 1, 80>>(),
        half_tile_info<HalfTile<32, 1, 1, 1, 1, 1, 8, 1, 80>>(),
    };
    *count = sizeof list / sizeof list[0];
    return list;
}

}  // namespace nmspmm
