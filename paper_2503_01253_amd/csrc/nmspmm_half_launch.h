// Launch of one instantiation of the tiled kernel (included by the units that
// instantiate it).
#ifndef NMSPMM_HALF_LAUNCH_H
#define NMSPMM_HALF_LAUNCH_H

#include "nmspmm_half_tile.h"
#include "nmspmm_half_tiles.h"

namespace nmspmm {

template <class C>
hipError_t launch_half_tile(const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.tiles_m * a.tiles_n * a.splits)), block(C::NT);
    if (bf16 && vec) hipLaunchKernelGGL((nm_half_tile_kernel<bf16_t, C, true>), grid, block, 0, stream, a);
    else if (bf16) hipLaunchKernelGGL((nm_half_tile_kernel<bf16_t, C, false>), grid, block, 0, stream, a);
    else if (vec) hipLaunchKernelGGL((nm_half_tile_kernel<f16_t, C, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((nm_half_tile_kernel<f16_t, C, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <class C>
HalfTileInfo half_tile_info()
{
    return {C::MI, C::CT, C::WK, C::BM, C::BN, C::KMAX, launch_half_tile<C>};
}

}  // namespace nmspmm

#endif
