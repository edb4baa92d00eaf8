// The kernel of few rows: its instantiations.
#include "nmspmm_half_short.h"
#include "nmspmm_half_tiles.h"

namespace nmspmm {
namespace {

template <class T, int MI>
hipError_t launch(const HalfShortArgs &a, bool wide, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.n / MI)), block(HS_NT);
    if (wide) hipLaunchKernelGGL((nm_half_short_kernel<T, MI, HS_SLOT_WIDE>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((nm_half_short_kernel<T, MI, HS_SLOT>), grid, block, 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_half_short(int MI, const HalfShortArgs &a, bool bf16, bool wide, hipStream_t stream)
{
    if (MI == 32) return bf16 ? launch<bf16_t, 32>(a, wide, stream) : launch<f16_t, 32>(a, wide, stream);
    return bf16 ? launch<bf16_t, 16>(a, wide, stream) : launch<f16_t, 16>(a, wide, stream);
}

}  // namespace nmspmm
