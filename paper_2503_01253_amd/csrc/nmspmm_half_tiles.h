// Host-side list of the tiled kernel's instantiations.
#ifndef NMSPMM_HALF_TILES_H
#define NMSPMM_HALF_TILES_H

#include <hip/hip_runtime_api.h>

namespace nmspmm {

struct HalfTileArgs;

struct HalfTileInfo {
    int MI, CT, WK, BM, BN, kmax;
    hipError_t (*launch)(const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream);
};

// one list per matrix-instruction shape and columns of a gather
const HalfTileInfo *half_tiles_32x1(int *count);
const HalfTileInfo *half_tiles_32x2(int *count);
const HalfTileInfo *half_tiles_16(int *count);

}  // namespace nmspmm

#endif
