// Host-side list of the tiled kernel's shapes.
#ifndef NMSPMM_HALF_TILES_H
#define NMSPMM_HALF_TILES_H

#include <hip/hip_runtime_api.h>

namespace nmspmm {

struct HalfTileArgs;
struct HalfShortArgs;

// X(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS KB, loads that need no alignment too)
#define NMSPMM_HALF_TILES(X)                              \
    X(32, 1, 2, 4, 1, 4, 1, 2, 1, 80, 0) /* 128 x 256 */     \
    X(32, 1, 1, 4, 1, 4, 1, 2, 2, 80, 0) /* 128 x 128 */     \
    X(32, 1, 1, 2, 1, 4, 2, 1, 2, 80, 1) /* 64 x 128 */      \
    X(32, 1, 1, 2, 1, 2, 4, 1, 2, 80, 0) /* 64 x 64 */       \
    X(32, 1, 1, 1, 1, 2, 4, 1, 2, 80, 0) /* 32 x 64 */       \
    X(32, 1, 1, 1, 1, 1, 8, 1, 2, 80, 0) /* 32 x 32 */       \
    X(32, 2, 1, 4, 1, 4, 1, 2, 1, 80, 0) /* 128 x 256 */     \
    X(32, 2, 1, 2, 2, 2, 1, 2, 2, 80, 0) /* 128 x 128 */     \
    X(32, 2, 1, 2, 1, 2, 2, 2, 2, 80, 0) /* 64 x 128 */      \
    X(32, 2, 1, 1, 1, 1, 8, 1, 2, 80, 0) /* 32 x 64 */       \
    X(16, 1, 2, 8, 1, 4, 1, 2, 1, 80, 1) /* 128 x 128 */     \
    X(16, 1, 2, 4, 1, 2, 4, 1, 1, 80, 0) /* 64 x 64 */       \
    X(16, 1, 2, 2, 1, 1, 8, 1, 2, 80, 0) /* 32 x 32 */

// A stage of 1 to 4 operands a wave.
constexpr int HALF_MAX_QS = 4;

// Launches tile `tile` of the list above with stages of QS operands a wave, one unit each.
hipError_t launch_half_q1(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream);
hipError_t launch_half_q2(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream);
hipError_t launch_half_q3(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream);
hipError_t launch_half_q4(int tile, const HalfTileArgs &a, bool bf16, bool vec, hipStream_t stream);

// Launches the kernel of few rows (nmspmm_half_short.h), with its wide slots or the others.
hipError_t launch_half_short(int MI, const HalfShortArgs &a, bool bf16, bool wide, hipStream_t stream);

}  // namespace nmspmm

#endif
