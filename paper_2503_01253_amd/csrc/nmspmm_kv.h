// Shared by the units of the paged cache: the device view of the cache, its
// addressing, and the joining of partial softmax results (device code).
#ifndef NMSPMM_KV_H
#define NMSPMM_KV_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "nmspmm_dtype.h"
#include "nmspmm_serve.h"

namespace nmspmm {

// Quotient by a divisor fixed on the host, of any n < 2^31: one high product,
// an addition that cannot overflow and a shift (the round-up method).
struct FastDiv {
    uint32_t mul, shift, d;
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(mul, n) + n) >> shift; }
};

inline FastDiv fast_div(uint32_t d)     // 1 <= d < 2^31
{
    uint32_t shift = 0;
    while ((1u << shift) < d) ++shift;
    const uint64_t one = 1;
    return {(uint32_t)(((one << 32) * ((one << shift) - d)) / d + 1), shift, d};
}

// The cache as the kernels see it.  row(p): the page of position p through
// the sequence's row of the table, or -1 where the table names no page of the
// cache.  Offsets are 64-bit: a cache holds more than 2^31 elements.
struct Pages {
    const int32_t *table;
    int64_t table_stride;
    int64_t pages;
    int64_t ks[3], vs[3];
    FastDiv size;
};

struct Place {
    int64_t page;
    int32_t slot;
    bool held;
};

__device__ __forceinline__ Place place_of(const Pages &c, const int32_t *row, int pos)
{
    const uint32_t at = c.size.div((uint32_t)pos);
    const int32_t page = row[at];
    return {page, pos - (int32_t)(at * c.size.d), page >= 0 && page < c.pages};
}

// (a, b) turned by the angle of cos c and sin s.  Spelled with fused
// multiply-adds whose fp32 results are kept (fp16's rounding is not fused into
// them), so that every kernel rounds alike.
__device__ __forceinline__ void turn_pair(float &a, float &b, float c, float s)
{
    float x = fmaf(a, c, -(b * s)), y = fmaf(a, s, b * c);
#ifdef __HIP_DEVICE_COMPILE__
    asm("" : "+v"(x), "+v"(y));
#endif
    a = x;
    b = y;
}

// The first (or the second) of a pair alone, rounded as turn_pair rounds it.
// s: minus the sine for the first.
__device__ __forceinline__ float turn_one(float own, float other, float c, float s, bool second)
{
    float y = second ? fmaf(other, s, own * c) : fmaf(own, c, other * s);
#ifdef __HIP_DEVICE_COMPILE__
    asm("" : "+v"(y));
#endif
    return y;
}

constexpr float NEG_INF = -__builtin_inff();

// The reference a running maximum stands for: scores are taken relative to
// it, and where nothing has been seen (minus infinity) relative to 0, so that
// no difference of two infinities arises.
__device__ __forceinline__ float softmax_ref(float m) { return m == NEG_INF ? 0.f : m; }

// The sum of x over the LPT lanes of a team, in every one of them.
template <int LPT>
__device__ __forceinline__ float lanes_sum(float x)
{
    auto dpp = [](float v, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value,
                                                                     0xf, 0xf, false));
    };
    x += dpp(x, std::integral_constant<int, 0xb1>{});                          // lane ^ 1
    x += dpp(x, std::integral_constant<int, 0x4e>{});                          // lane ^ 2
    if constexpr (LPT >= 8) x += dpp(x, std::integral_constant<int, 0x141>{});  // the other four of eight
    if constexpr (LPT >= 16) x += dpp(x, std::integral_constant<int, 0x140>{}); // the other eight of sixteen
    if constexpr (LPT >= 32) x += __shfl_xor(x, 16);
    if constexpr (LPT >= 64) x += __shfl_xor(x, 32);
    return x;
}

struct AttendArgs {
    Pages c;
    const void *q, *k, *v;
    void *out;
    float *lse, *part_acc;
    float2 *part_ml;
    const int32_t *lengths;
    int64_t qs[2], os[2];
    int32_t cap, window;        // cap: the smaller of max_length and the table's positions
    int32_t heads, group, gtiles, dim, splits, chunk;
    float scale2;               // scale * log2(e): exponentials are powers of 2
    nmspmm_dtype_t io;
    bool q_vec;                 // the queries' rows start on 16 bytes
};

// One workgroup's work: a tile of query heads of one cache head of one
// sequence, and its chunk of the positions.
struct AttendTask {
    int64_t seq, first_head;    // first_head: of the tile, among the query heads
    int32_t head, split, heads_in_tile, begin, end;
};

__device__ __forceinline__ AttendTask attend_task(const AttendArgs &p, uint32_t id, int GT)
{
    AttendTask t;
    const uint32_t gt = id % p.gtiles;
    id /= p.gtiles;
    t.head = id % p.heads;
    id /= p.heads;
    t.split = id % p.splits;
    t.seq = id / p.splits;
    t.first_head = (int64_t)t.head * p.group + gt * GT;
    t.heads_in_tile = p.group - (int)gt * GT < GT ? p.group - (int)gt * GT : GT;
    const int32_t len = p.lengths[t.seq] < p.cap ? p.lengths[t.seq] : p.cap;
    const int32_t first = p.window > 0 && len > p.window ? len - p.window : 0;
    const int64_t begin = first + (int64_t)t.split * p.chunk;
    t.begin = begin < len ? (int32_t)begin : (len > 0 ? len : 0);
    t.end = begin + p.chunk < len ? (int32_t)(begin + p.chunk) : len;
    return t;
}

// One query head's result: normalised into out (and lse) where the sequence
// was not split, else the unnormalised sums with their maximum and sum.
// x: the value of dimension d relative to maximum m (in powers of 2), l: the
// sum of the weights.
__device__ __forceinline__ void attend_store(const AttendArgs &p, const AttendTask &t, int64_t head, int d, float x,
                                             float m, float l)
{
    const int64_t row = t.seq * ((int64_t)p.heads * p.group) + head;
    if (p.splits == 1) {
        const float y = l == 0.f ? 0.f : x / l;
        const int64_t at = t.seq * p.os[0] + head * p.os[1] + d;
        if (p.io == NMSPMM_F32) static_cast<float *>(p.out)[at] = y;
        else if (p.io == NMSPMM_BF16) static_cast<bf16_t *>(p.out)[at] = from_f32<bf16_t>(y);
        else static_cast<f16_t *>(p.out)[at] = from_f32<f16_t>(y);
        if (d == 0 && p.lse) p.lse[row] = l == 0.f ? NEG_INF : 0.69314718056f * (m + log2f(l));
    } else {
        p.part_acc[(row * p.splits + t.split) * p.dim + d] = x;
        if (d == 0) p.part_ml[row * p.splits + t.split] = make_float2(m, l);
    }
}

// nmspmm_kv_mfma.hip: an fp16 cache with fp16 queries or a bf16 cache with any,
// rows of whole 16-byte pieces, at most 256 dimensions; tiles of 16 heads.
constexpr int ATTEND_MFMA_HEADS = 16;
void launch_attend_mfma(const AttendArgs &p, nmspmm_dtype_t cache, unsigned groups, hipStream_t stream);

}  // namespace nmspmm

#endif
