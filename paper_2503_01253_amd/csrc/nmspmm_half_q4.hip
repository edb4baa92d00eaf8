// The tiled kernel with stages of 4 operands a wave.
#include "nmspmm_half_launch.h"

namespace nmspmm {

hipError_t launch_half_q4(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream)
{
    return launch_half<4>(tile, a, bf16, vec, stream);
}

}  // namespace nmspmm
