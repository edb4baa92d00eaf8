// The tiled kernel with stages of 2 operands a wave.
#include "nmspmm_half_launch.h"

namespace nmspmm {

hipError_t launch_half_q2(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream)
{
    return launch_half<2>(tile, a, bf16, vec, stream);
}

}  // namespace nmspmm
