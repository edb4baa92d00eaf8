// The sparse product with a 4-bit weight for more than 16 rows: its instances.
#include <hip/hip_runtime.h>

#include "nmspmm_mx4_tile.h"

namespace nmspmm {
namespace {

template <class T, int MT, int CT, int WC, int D>
void launch_of(const Mx4Args &p, const dim3 &grid, hipStream_t stream)
{
    if (p.vec) hipLaunchKernelGGL((nm_mx4_wide_kernel<T, MT, CT, WC, D, true>), grid, dim3(MX4_NT), 0, stream, p);
    else hipLaunchKernelGGL((nm_mx4_wide_kernel<T, MT, CT, WC, D, false>), grid, dim3(MX4_NT), 0, stream, p);
}

template <class T, int MT, int CT>
void launch(int WC, int D, const Mx4Args &p, const dim3 &grid, hipStream_t stream)
{
    if (WC == 8) launch_of<T, MT, CT, 8, 1>(p, grid, stream);
    else if (D == 1) launch_of<T, MT, CT, 4, 1>(p, grid, stream);
    else if (D == 2) launch_of<T, MT, CT, 4, 2>(p, grid, stream);
    else launch_of<T, MT, CT, 4, 4>(p, grid, stream);
}

template <class T>
void launch_tiles(int MT, int CT, int WC, int D, const Mx4Args &p, const dim3 &grid, hipStream_t stream)
{
    if (MT == 2) {
        if (CT == 1) launch<T, 2, 1>(WC, D, p, grid, stream);
        else if (CT == 2) launch<T, 2, 2>(WC, D, p, grid, stream);
        else launch<T, 2, 4>(WC, D, p, grid, stream);
    } else {
        if (CT == 1) launch<T, 4, 1>(WC, D, p, grid, stream);
        else if (CT == 2) launch<T, 4, 2>(WC, D, p, grid, stream);
        else launch<T, 4, 4>(WC, D, p, grid, stream);
    }
}

}  // namespace

void launch_mx4_wide(int MT, int CT, int WC, int D, bool bf16, const Mx4Args &p, const dim3 &grid, hipStream_t stream)
{
    if (bf16) launch_tiles<bf16_t>(MT, CT, WC, D, p, grid, stream);
    else launch_tiles<f16_t>(MT, CT, WC, D, p, grid, stream);
}

}  // namespace nmspmm
