// Host-side list of the tiled kernel's shapes.
#ifndef NMSPMM_HALF_TILES_H
#define NMSPMM_HALF_TILES_H

#include <hip/hip_runtime_api.h>

namespace nmspmm {

struct HalfTileArgs;
struct HalfShortArgs;

// X(MI, CT, NG, RT, WR, WC, WK, NB, AD, LDS KB, loads that need no alignment too)
//
// Of tiles that cost the same by the estimate the first is taken.  So is CT = 2,
// one gather for two operands, where V is a multiple of 64 and tiles are 128 x
// 256: faster on all of 50 shapes (4096^3 at 16:32 101 us and 107 with CT = 1, at
// 4:32 54.6 and 56.0, 2048 x 4096 x 11008 at 8:32 96 and 99).  In smaller tiles
// its longer waves lost as much as they gained: 128 x 128 within 2 % either way,
// 64 x 128 slower wherever it was the best size (512 x 2048 x 2048 16.1 and 14.7).
#define NMSPMM_HALF_TILES(X)                              \
    X(32, 2, 1, 4, 1, 4, 1, 2, 1, 80, 0) /* 128 x 256 */     \
    X(32, 1, 2, 4, 1, 4, 1, 2, 1, 80, 0) /* 128 x 256 */     \
    X(32, 1, 1, 4, 1, 4, 1, 2, 2, 80, 0) /* 128 x 128 */     \
    X(32, 1, 1, 2, 1, 4, 2, 1, 2, 80, 1) /* 64 x 128 */      \
    X(32, 1, 1, 2, 1, 2, 4, 1, 2, 80, 0) /* 64 x 64 */       \
    X(32, 1, 1, 1, 1, 2, 4, 1, 2, 80, 0) /* 32 x 64 */       \
    X(32, 1, 1, 1, 1, 1, 8, 1, 2, 80, 0) /* 32 x 32 */       \
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
