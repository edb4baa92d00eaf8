// Launches of the tiled kernel with stages of one length (included by the
// units that instantiate them).
#ifndef NMSPMM_HALF_LAUNCH_H
#define NMSPMM_HALF_LAUNCH_H

#include "nmspmm_half_tile.h"
#include "nmspmm_half_tiles.h"

namespace nmspmm {

template <class T, class C, int QS, bool ANY>
hipError_t launch_half_tile(const HalfTileArgs &a, bool vec, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.tiles_m * a.tiles_n * a.splits)), block(C::NT);
    if (vec) hipLaunchKernelGGL((nm_half_tile_kernel<T, C, QS, true>), grid, block, 0, stream, a);
    else if constexpr (ANY) hipLaunchKernelGGL((nm_half_tile_kernel<T, C, QS, false>), grid, block, 0, stream, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

template <int QS>
hipError_t launch_half(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream)
{
    int at = 0;
#define NMSPMM_HALF_CASE(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS, ANY)                                                   \
    if (tile == at++)                                                                                                \
        return bf16 ? launch_half_tile<bf16_t, HalfTile<MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS>, QS, ANY>(a, vec, stream) \
                    : launch_half_tile<f16_t, HalfTile<MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS>, QS, ANY>(a, vec, stream);
    NMSPMM_HALF_TILES(NMSPMM_HALF_CASE)
#undef NMSPMM_HALF_CASE
    return hipErrorInvalidValue;
}

}  // namespace nmspmm

#endif
