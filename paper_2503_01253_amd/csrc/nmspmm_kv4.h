// Shared by the units of the 4-bit cache: how a page holds its rows, and the
// device view of the cache.
//
// A page holds, head after head, a block: the codes of its keys, those of its
// values, the keys' scales and the values' scales, each part on 16 bytes, so
// that all of a head's tokens lie in one piece (dim 128, 16 tokens: 2176 bytes).
// A row of dim dimensions has G = ceil(dim/32) groups and 4 G words of eight
// codes; word D holds the dimensions 8D to 8D+7.
//   keys     slot after slot; the words of a row in the order 4 c + g -> g G + c
//            (c: the group, g: the word within it), so that the lanes with
//            g = 0 to 3 of a matrix instruction, which each take word g of
//            every group, read G words in one piece
//   values   four slots together: word D of slots 4q to 4q+3 side by side (16
//            bytes), so that a lane reads the same dimensions of four tokens
//   scales   keys: a slot's G bytes, as many bytes apart as the next power of
//            2; values: group c of slots 4q to 4q+3 side by side (4 bytes)
#ifndef NMSPMM_KV4_H
#define NMSPMM_KV4_H

#include <cstdint>

#include "nmspmm_kv.h"
#include "nmspmm_fp4.h"
#include "nmspmm_mx4.h"

namespace nmspmm {

struct Kv4Layout {
    int64_t v_at, ks_at, vs_at, block;      // of a head's block: where its parts start, and its bytes
    int32_t G, sp;                          // groups of a row, bytes from one slot's key scales to the next's

    __host__ __device__ __forceinline__ int64_t k_word(int64_t slot, int D) const
    {
        return slot * (16 * G) + ((D & 3) * G + (D >> 2)) * 4;
    }
    __host__ __device__ __forceinline__ int64_t v_word(int64_t slot, int D) const
    {
        return v_at + (slot >> 2) * (64 * G) + D * 16 + (slot & 3) * 4;
    }
    __host__ __device__ __forceinline__ int64_t k_scale(int64_t slot, int c) const { return ks_at + slot * sp + c; }
    __host__ __device__ __forceinline__ int64_t v_scale(int64_t slot, int c) const
    {
        return vs_at + (slot >> 2) * (4 * G) + c * 4 + (slot & 3);
    }
};

inline Kv4Layout kv4_layout(int64_t page_size, int64_t dim)
{
    Kv4Layout l{};
    l.G = (int32_t)((dim + 31) / 32);
    for (l.sp = 1; l.sp < l.G;) l.sp *= 2;
    const int64_t quads = (page_size + 3) / 4;
    l.v_at = page_size * 16 * l.G;
    l.ks_at = l.v_at + quads * 64 * l.G;
    l.vs_at = (l.ks_at + page_size * l.sp + 15) / 16 * 16;
    l.block = (l.vs_at + quads * 4 * l.G + 15) / 16 * 16;
    return l;
}

// The cache as the kernels see it (its table is in a Pages).
struct Kv4Pages {
    unsigned char *pages;
    int64_t stride;
    Kv4Layout l;
    __device__ __forceinline__ unsigned char *block(int64_t page, int64_t head) const
    {
        return pages + page * stride + head * l.block;
    }
};

// nmspmm_kv4.hip: the sizes of a 4-bit cache as those of a 16-bit one, for the
// checks and plans that only look at sizes, and the checks of what it has of its own.
nmspmm_kv_cache_t kv4_sizes(const nmspmm_kv4_cache_t *c);
nmspmm_status_t check_kv4(const nmspmm_kv4_cache_t *c);
nmspmm_status_t check_kv4_pointers(const nmspmm_kv4_cache_t *c);
Kv4Pages kv4_view(const nmspmm_kv4_cache_t *c);

// nmspmm_kv4_mfma.hip: pages of whole fours of tokens, a head's block under 2^31
// bytes, at most 256 dimensions; tiles of ATTEND_MFMA_HEADS heads.
void launch_attend4_mfma(const AttendArgs &p, const Kv4Pages &f, int page_size, unsigned groups, hipStream_t stream);

}  // namespace nmspmm

#endif
