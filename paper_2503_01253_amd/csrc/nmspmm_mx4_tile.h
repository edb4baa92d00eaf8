// Kernels of the product with a 4-bit weight for few rows (device code), where
// V is a multiple of 16: bound by the weight's bytes and by latency.
//
// The packed weight holds B operands of v_mfma_f32_16x16x32 as its lanes read
// them: lane l has the eight codes of column l % 16 and compressed rows 8 (l / 16)
// and on, one word, of 32 compressed rows: a group, which is also what shares a
// scale.  A word becomes an operand of bf16 by four conversions that apply the
// scale; with fp16 rows, whose range the scales would leave, the codes are
// converted as they are and the group's sums are multiplied in fp32.
//   dense (N = M)   four groups of one column tile a lane's 16 bytes (a step);
//                   A's operands come straight from memory, 16 bytes a lane
//   sparse          one group of CT column tiles of one block a lane's 4 CT
//                   bytes; A's operands are gathered from LDS at the group's
//                   offsets, one gather for all CT tiles: up to 16 rows from rows
//                   as they lie in memory, eight 2-byte reads an operand; more,
//                   from a k-major copy, two transposed reads an operand
#ifndef NMSPMM_MX4_TILE_H
#define NMSPMM_MX4_TILE_H

#include "nmspmm_fp4.h"
#include "nmspmm_half_tile.h"

namespace nmspmm {

struct Mx4Args {
    const void *A;
    const unsigned char *vals, *scales;
    const uint16_t *offs;
    float *part;                // with split k: splits x m x n partial sums
    int64_t lda, m, n, k, first_row;
    int32_t w, N, M, V;
    int32_t steps;              // groups (dense: steps of four) of all of k
    int32_t splits, per_split;  // slices of k, for more than 16 rows (neighbouring workgroups: a slice's
                                // are on one XCD, which reads its part of A once), and the steps of one
    int32_t tiles;              // runs of CT column tiles (dense: column tiles)
    int32_t rows;               // rows of a workgroup, 16 MT at most
    int32_t chunk;              // sparse: groups of a chunk of A (a multiple of WK)
    int32_t pitch, slot;        // bytes of its rows in LDS, and of a slot (all of LDS: one chunk)
    bool vec;                   // A's rows start on 16 bytes and k is a multiple of 8
    HalfEpilogue epi;
};

constexpr int MX4_NW = 8, MX4_NT = 64 * MX4_NW;

template <class T>
__device__ __forceinline__ s16x8 mx4_operand(uint32_t w, float scale)
{
    uint32_t r[4];
    if constexpr (__is_same(T, bf16_t)) {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    } else {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 3));
    }
    return __builtin_bit_cast(s16x8, u32x4{r[0], r[1], r[2], r[3]});
}

// acc += A * B over one group of 32 compressed rows, MT operands of A.
template <class T, int MT>
__device__ __forceinline__ void mx4_group(const s16x8 (&a)[MT], uint32_t w, float scale, f32x4 (&acc)[MT])
{
    const s16x8 b = mx4_operand<T>(w, scale);
    if constexpr (__is_same(T, bf16_t)) {
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = half_mfma<T, 16>(a[t], b, acc[t]);
    } else {
        // the scale as a value: 2^-127 and NaN included
        const float s = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(2, scale, 0)[0];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const f32x4 sum = half_mfma<T, 16>(a[t], b, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(sum[e], s, acc[t][e]);
        }
    }
}

// What the epilogue reads for four columns of a row.
struct Mx4Ahead {
    float bias[4], mul[4], residual[4];
};

template <class O, bool VEC>
__device__ __forceinline__ void mx4_fetch_of(const HalfEpilogue &e, int64_t r, int64_t j, Mx4Ahead &a)
{
    if (e.bias) load_row<4, VEC>(e.bias + j, 4, a.bias);
    if (e.mul) load_row<4, VEC>(static_cast<const O *>(e.mul) + r * e.ld_mul + j, 4, a.mul);
    if (e.residual) load_row<4, VEC>(static_cast<const O *>(e.residual) + r * e.ld_residual + j, 4, a.residual);
}

template <class T>
__device__ __forceinline__ Mx4Ahead mx4_fetch(const HalfEpilogue &e, int64_t r, int64_t j)
{
    Mx4Ahead a{};
    if (e.f32) e.vec ? mx4_fetch_of<float, true>(e, r, j, a) : mx4_fetch_of<float, false>(e, r, j, a);
    else e.vec ? mx4_fetch_of<T, true>(e, r, j, a) : mx4_fetch_of<T, false>(e, r, j, a);
    return a;
}

// The epilogue of four sums.
template <class T>
__device__ __forceinline__ void mx4_emit(const HalfEpilogue &e, int64_t r, int64_t j, const float (&sum)[4],
                                         const Mx4Ahead &a)
{
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = e.alpha * sum[i] + (e.bias ? a.bias[i] : 0.f);
    if (e.act != NMSPMM_HALF_ACT_NONE) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {       // (one copy of the activations' code)
            float v = half_act(y[0], e.act);
            y[0] = y[1], y[1] = y[2], y[2] = y[3], y[3] = v;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (e.mul) y[i] *= a.mul[i];
        if (e.residual) y[i] += a.residual[i];
    }
    if (e.f32) {
        float *dst = static_cast<float *>(e.C) + r * e.ldc + j;
        e.vec ? store_row<4, true>(dst, 4, y) : store_row<4, false>(dst, 4, y);
    } else {
        T *dst = static_cast<T *>(e.C) + r * e.ldc + j;
        e.vec ? store_row<4, true>(dst, 4, y) : store_row<4, false>(dst, 4, y);
    }
}

// Up to 16 rows: what the epilogue reads for a thread's first output, asked for at the
// kernel's start (for one row: all of it; the last reads of a kernel that latency bounds:
// 1 x 4096 x 4096, dense, 5.4 -> 4.8 us).
struct Mx4First {
    float bias, mul, residual;
};

template <class T, int COLS>
__device__ __forceinline__ Mx4First mx4_first(const Mx4Args &p, int64_t row0, int64_t col0, int rows)
{
    Mx4First a{0.f, 1.f, 0.f};
    const int row = threadIdx.x / COLS;
    const int64_t r = row0 + row, j = col0 + threadIdx.x % COLS;
    if (row >= rows || j >= p.n) return a;
    if (p.epi.bias) a.bias = p.epi.bias[j];
    if (p.epi.mul) {
        const int64_t at = r * p.epi.ld_mul + j;
        a.mul = p.epi.f32 ? static_cast<const float *>(p.epi.mul)[at] : to_f32(static_cast<const T *>(p.epi.mul)[at]);
    }
    if (p.epi.residual) {
        const int64_t at = r * p.epi.ld_residual + j;
        a.residual = p.epi.f32 ? static_cast<const float *>(p.epi.residual)[at]
                               : to_f32(static_cast<const T *>(p.epi.residual)[at]);
    }
    return a;
}

// half_store with those.
template <class O>
__device__ __forceinline__ void mx4_store(const HalfEpilogue &e, int64_t i, int64_t j, float sum, const Mx4First &a)
{
    float y = e.alpha * sum;
    if (e.bias) y += a.bias;
    y = half_act(y, e.act);
    if (e.mul) y *= a.mul;
    if (e.residual) y += a.residual;
    static_cast<O *>(e.C)[i * e.ldc + j] = from_f32<O>(y);
}

// The sums of the WK waves that share columns, added in their order, and the
// epilogue (or, with k in slices, the slice's partial sums: more than 16 rows only).  Wave wk * WC + wc holds
// columns wc * CT * 16 and on; red holds MX4_NW * CT * MT * 256 floats.  Up to 16 rows
// one output a thread, more than 16 four columns, MX4_U times at once (64 x 4096 at k =
// 512 one after another 15 us, so 8.4; 1 x 4096 x 11008, dense, 7.2 and so 9.2).
constexpr int MX4_U = 4;

template <class T, int MT, int CT, int WC>
__device__ __forceinline__ void mx4_finish(const Mx4Args &p, float *red, const f32x4 (&acc)[CT][MT], int64_t row0,
                                           int64_t col0, int rows, bool split, const Mx4First &ahead)
{
    constexpr int WK = MX4_NW / WC, COLS = WC * CT * 16;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    lds_sync();
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[(((wave * CT + c) * MT + t) * 4 + e) * 64 + lane] = acc[c][t][e];
    lds_sync();
    if constexpr (MT == 1) {
        for (int i = tid; i < rows * COLS; i += MX4_NT) {
            const int row = i / COLS, col = i % COLS;
            const float *x = red + ((col / 16) * 4 + row % 4) * 64 + row / 4 * 16 + col % 16;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < WK; ++k) sum += x[k * (WC * CT * 256)];
            const int64_t r = row0 + row, j = col0 + col;
            if (j >= p.n) continue;
            if (i == tid) {
                if (p.epi.f32) mx4_store<float>(p.epi, r, j, sum, ahead);
                else mx4_store<T>(p.epi, r, j, sum, ahead);
            } else if (p.epi.f32) half_store<float>(p.epi, r, j, sum);
            else half_store<T>(p.epi, r, j, sum);
        }
    } else {
        const int64_t part = split ? ((int64_t)(blockIdx.x % p.splits) * p.m + row0) * p.n : 0;
        for (int first = tid; first < rows * COLS / 4; first += MX4_NT * MX4_U) {
            Mx4Ahead a[MX4_U];
#pragma unroll
            for (int u = 0; u < MX4_U; ++u) {
                const int i = first + u * MX4_NT, row = i * 4 / COLS;
                const int64_t j = col0 + i * 4 % COLS;
                if (!split && row < rows && j < p.n) a[u] = mx4_fetch<T>(p.epi, row0 + row, j);
            }
#pragma unroll
            for (int u = 0; u < MX4_U; ++u) {
                const int i = first + u * MX4_NT, row = i * 4 / COLS, col = i * 4 % COLS;
                const int64_t j = col0 + col;
                if (row >= rows || j >= p.n) continue;
                const float *x = red + (((col / 16) * MT + row / 16) * 4 + row % 4) * 64 + row % 16 / 4 * 16 + col % 16;
                float sum[4] = {};
#pragma unroll
                for (int k = 0; k < WK; ++k) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(x + k * (WC * CT * MT * 256));
#pragma unroll
                    for (int q = 0; q < 4; ++q) sum[q] += v[q];
                }
                if (split) *reinterpret_cast<f32x4 *>(p.part + part + row * p.n + j) = f32x4{sum[0], sum[1], sum[2], sum[3]};
                else mx4_emit<T>(p.epi, row0 + row, j, sum, a[u]);
            }
        }
    }
}

// Dense.  A workgroup owns CT column tiles and 16 MT rows; its eight waves take
// the steps of (a slice of) k in turn, D of them on their way.  VEC: A's rows
// start on 16 bytes and k is a multiple of 8.  (1 x 4096 x 11008, CT = 3: D = 2 7.2 us,
// 3.3 TB/s, D = 3 8.4, D = 4 8.3; CT = 4 keeps four registers in memory; 1 x 4096 x 4096, CT = 1: 4.8, 5.6, 5.6.  Lanes of rows
// past the last that load nothing: 7.6 and 5.4, for their branches.)
template <class T, int MT, int CT, int D, bool VEC>
__global__ __launch_bounds__(MX4_NT, MT == 1 && VEC ? 4 : 2) void nm_mx4_dense_kernel(Mx4Args p)
{
    __shared__ __align__(16) float red[MX4_NW * CT * MT * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int64_t row0 = p.first_row + (int64_t)blockIdx.y * p.rows;
    const int rows = (int)min64(p.rows, p.m - row0);
    const bool split = MT > 1 && p.splits > 1;
    const int column = split ? blockIdx.x / p.splits : blockIdx.x, slice = split ? blockIdx.x - column * p.splits : 0;
    const int first = slice * p.per_split, last = min(first + p.per_split, p.steps) - 1;
    const unsigned char *vals[CT], *scales[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int64_t tile = min(column * CT + c, p.tiles - 1);
        vals[c] = p.vals + tile * p.steps * 1024 + lane * 16;
        scales[c] = p.scales + tile * p.steps * 64 + col * 4;
    }
    const T *a_row[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) a_row[t] = static_cast<const T *>(p.A) + (row0 + min(t * 16 + col, rows - 1)) * p.lda;

    const int64_t col0 = (int64_t)column * (CT * 16);
    const Mx4First ahead = MT == 1 ? mx4_first<T, CT * 16>(p, row0, col0, rows) : Mx4First{};
    u32x4 rv[D][CT];
    uint32_t rs[D][CT];
    s16x8 ra[D][4][MT];
    auto load = [&](int i, int step) {
        const int64_t s = min(step, last);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            rv[i][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vals[c] + s * 1024));
            rs[i][c] = *reinterpret_cast<const uint32_t *>(scales[c] + s * 64);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int64_t at = s * 128 + g * 32 + grp * 8;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (VEC) {
                    ra[i][g][t] = *reinterpret_cast<const s16x8 *>(a_row[t] + min64(at, p.k - 8));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        ra[i][g][t][j] = at + j < p.k ? __builtin_bit_cast(short, a_row[t][at + j]) : (short)0;
                }
            }
        }
    };
    f32x4 acc[CT][MT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int i, int step) {
        if (step > last) return;
        if (VEC && (int64_t)step * 128 + 128 > p.k) {       // columns past k: zeros
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    if ((int64_t)step * 128 + g * 32 + grp * 8 >= p.k) ra[i][g][t] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            mx4_group<T, MT>(ra[i][0], rv[i][c][0], mx4_scale<0>(rs[i][c]), acc[c]);
            mx4_group<T, MT>(ra[i][1], rv[i][c][1], mx4_scale<1>(rs[i][c]), acc[c]);
            mx4_group<T, MT>(ra[i][2], rv[i][c][2], mx4_scale<2>(rs[i][c]), acc[c]);
            mx4_group<T, MT>(ra[i][3], rv[i][c][3], mx4_scale<3>(rs[i][c]), acc[c]);
        }
    };
#pragma unroll
    for (int i = 0; i < D; ++i) load(i, first + wave + i * MX4_NW);
    for (int step = first + wave; step <= last; step += D * MX4_NW) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            compute(i, step + i * MX4_NW);
            load(i, step + (i + D) * MX4_NW);
        }
    }
    mx4_finish<T, MT, CT, 1>(p, red, acc, row0, col0, rows, split, ahead);
}

// The first column of A that group s can meet.
__device__ __forceinline__ int64_t mx4_base(const Mx4Args &p, int s)
{
    return (int64_t)((uint32_t)s * 32u / (uint32_t)p.N) * p.M;
}

// The columns of A that a chunk of groups from s on, or up to s, is loaded from and to.
__device__ __forceinline__ int64_t mx4_chunk_base(const Mx4Args &p, int s) { return mx4_base(p, s) & ~(int64_t)7; }
__device__ __forceinline__ int64_t mx4_chunk_end(const Mx4Args &p, int s)
{
    return min64(p.k, ((int64_t)(((uint32_t)s * 32u - 1u) / (uint32_t)p.N) + 1) * p.M);
}

// Zeros in the places of compressed rows past the last.
template <int MT>
__device__ __forceinline__ void mx4_pad(const Mx4Args &p, int step, int grp, s16x8 (&a)[MT])
{
    if (step < p.steps - 1 || p.w % 32 == 0) return;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (grp * 8 + j >= p.w % 32)
#pragma unroll
            for (int t = 0; t < MT; ++t) a[t][j] = 0;
}

__device__ __forceinline__ float mx4_scale_at(uint32_t four, int i)
{
    return i == 0 ? mx4_scale<0>(four) : i == 1 ? mx4_scale<1>(four) : i == 2 ? mx4_scale<2>(four) : mx4_scale<3>(four);
}

// Sparse, up to 16 rows.  WC waves take neighbouring runs of CT column tiles, and
// the MX4_NW / WC waves that share columns the groups of every chunk of A in turn, D
// of them on their way.  A_s: the rows of A over the chunk's columns, as they lie
// in memory: all of them, or in two slots, where the next chunk lands meanwhile.
template <class T, int CT, int WC, int D, int LDS>
__global__ __launch_bounds__(MX4_NT, LDS <= 80 * 1024 ? 4 : 2) void nm_mx4_sparse_kernel(Mx4Args p)
{
    constexpr int WK = MX4_NW / WC, SP = CT;
    static_assert(MX4_NW * CT * 1024 <= LDS, "the joining of the waves");
    __shared__ __align__(256) unsigned char lds[LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4, wc = wave % WC, wk = wave / WC;
    const int64_t row0 = p.first_row + (int64_t)blockIdx.y * p.rows;
    const int rows = (int)min64(p.rows, p.m - row0);
    const int column = blockIdx.x, end = p.steps;
    const int64_t tile = min(column * WC + wc, p.tiles - 1);
    const unsigned char *vals = p.vals + tile * p.steps * (256 * CT) + lane * (4 * CT);
    const unsigned char *scales = p.scales + tile * p.steps * (16 * SP) + col * SP;
    const unsigned char *offs = reinterpret_cast<const unsigned char *>(p.offs) +
                                (tile * (CT * 16) / p.V) * p.steps * 64 + grp * 16;

    const int64_t col0 = (int64_t)column * (WC * CT * 16);
    const Mx4First ahead = mx4_first<T, WC * CT * 16>(p, row0, col0, rows);
    uint32_t rv[D][CT], rs[D];
    u32x4 ro[D];
    auto load = [&](int i, int step) {
        const int64_t s = min(step, end - 1);
        __builtin_memcpy(rv[i], __builtin_assume_aligned(vals + s * (256 * CT), 4 * CT), 4 * CT);
        uint32_t four = 0;
        __builtin_memcpy(&four, __builtin_assume_aligned(scales + s * (16 * SP), SP), SP);
        rs[i] = four;
        ro[i] = *reinterpret_cast<const u32x4 *>(offs + s * 64);
    };

    // ---- A ----
    const T *A = static_cast<const T *>(p.A) + row0 * p.lda;
    const __amdgpu_buffer_rsrc_t a_rsrc = make_rsrc(A, p.vec ? (uint32_t)(((rows - 1) * p.lda + p.k) * 2) : 0u);
    auto load_a = [&](int s0, int slot) {
        const int s1 = min(s0 + p.chunk, end);
        const int64_t c0 = mx4_chunk_base(p, s0);
        const int cols = (int)(mx4_chunk_end(p, s1) - c0);
        unsigned char *dst = lds + slot * p.slot;
        if (p.vec) {
            const int pieces = (cols * 2 + 1023) / 1024;
            for (int x = wave; x < rows * pieces; x += MX4_NW) {
                const int row = x / pieces, at = (x - row * pieces) * 1024;
                if (at + lane * 16 < cols * 2)
                    lds_dma<16>(a_rsrc, dst + row * p.pitch + at,
                                (uint32_t)((row * p.lda + c0) * 2 + at + lane * 16));
            }
        } else {
            if constexpr (NMSPMM_POISON_LDS) {      // (as lds_dma does)
                for (int row = wave; row < rows; row += MX4_NW)
                    for (int c = lane; c < cols; c += 64)
                        *reinterpret_cast<uint16_t *>(dst + row * p.pitch + c * 2) = (uint16_t)~0u;
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));  // lgkmcnt(0)
            }
            for (int row = wave; row < rows; row += MX4_NW)
                for (int c = lane; c < cols; c += 64)
                    *reinterpret_cast<T *>(dst + row * p.pitch + c * 2) = A[row * p.lda + c0 + c];
        }
    };

    f32x4 acc[CT][1];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c][0] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (rows past the last read the last: their outputs are not stored)
    const int a_row = min(col, rows - 1) * p.pitch;

    auto compute = [&](int i, int step, int64_t c0, int slot) {
        if (step >= end) return;
        const int base = slot * p.slot + a_row + (int)(mx4_base(p, step) - c0) * 2;
        s16x8 a[1];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = base + (int)(j < 4 ? ro[i][j] & 0xffffu : ro[i][j - 4] >> 16);
            a[0][j] = *reinterpret_cast<const short *>(lds + at);
        }
        mx4_pad<1>(p, step, grp, a);
#pragma unroll
        for (int c = 0; c < CT; ++c) mx4_group<T, 1>(a, rv[i][c], mx4_scale_at(rs[i], c), acc[c]);
    };

    load_a(0, 0);
#pragma unroll
    for (int i = 0; i < D; ++i) load(i, wk + i * WK);
    // every wave takes the same number of groups (the last may be none), so
    // that all meet at the chunks' ends
    int slot = 1, chunk_end = 0;
    int64_t c0 = 0;
    for (int s0 = 0; s0 < end; s0 += D * WK) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int s = s0 + i * WK;
            if (s >= end) break;
            if (s == chunk_end) {       // a chunk is whole runs of WK groups
                stage_sync();
                slot ^= 1;
                c0 = mx4_chunk_base(p, s);
                chunk_end = s + p.chunk;
                if (chunk_end < end) load_a(chunk_end, slot ^ 1);
            }
            compute(i, s + wk, c0, slot);
            load(i, s + wk + D * WK);
        }
    }
    mx4_finish<T, 1, CT, WC>(p, reinterpret_cast<float *>(lds), acc, row0, col0, rows, false, ahead);
}

// Columns of A that a slot of the kernel below holds, and its threads' blocks of A.
constexpr int MX4_NB = 2;
__host__ __device__ constexpr int mx4_wide_columns(int MT) { return MX4_NB * MX4_NT * 32 / (16 * MT); }

// Sparse, 16 MT rows.  As above, but that A_s holds columns: LDS row c has column c
// of the chunk, its 16 MT rows in granules of 16 (32 bytes) of which the t-th lies
// at place t ^ swizzle(c).  A slab comes through registers, NB blocks of 4 rows and 8
// columns a thread, transposed by byte permutes; the next two are on their way
// meanwhile.
template <class T, int MT, int CT, int WC, int D, bool VEC>
__global__ __launch_bounds__(MX4_NT, 2) void nm_mx4_wide_kernel(Mx4Args p)
{
    constexpr int WK = MX4_NW / WC, SP = CT, CHUNK = D * WK, BM = 16 * MT, PITCH = 2 * BM, SWZ = MT - 1;
    constexpr int SLOT = mx4_wide_columns(MT) * PITCH, NB = MX4_NB, AD = 2;
    static_assert((MT == 2 || MT == 4) && MX4_NW * CT * MT * 1024 <= 2 * SLOT, "the joining of the waves");
    __shared__ __align__(256) unsigned char lds[2 * SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4, wc = wave % WC, wk = wave / WC;
    const int64_t row0 = p.first_row + (int64_t)blockIdx.y * p.rows;
    const int rows = (int)min64(p.rows, p.m - row0);
    const int column = p.splits > 1 ? blockIdx.x / p.splits : blockIdx.x, slice = blockIdx.x - column * p.splits;
    const int first = slice * p.per_split, end = min(first + p.per_split, p.steps);
    const int64_t tile = min(column * WC + wc, p.tiles - 1);
    const unsigned char *vals = p.vals + tile * p.steps * (256 * CT) + lane * (4 * CT);
    const unsigned char *scales = p.scales + tile * p.steps * (16 * SP) + col * SP;
    // a lane's two rows of the group's: 8 grp + r and 4 further, r = lane / 4 % 4
    const unsigned char *offs = reinterpret_cast<const unsigned char *>(p.offs) +
                                (tile * (CT * 16) / p.V) * p.steps * 64 + grp * 16 + (lane >> 2 & 3) * 4;

    const bool split = p.splits > 1;
    const int64_t col0 = (int64_t)column * (WC * CT * 16);
    uint32_t rv[D][CT], rs[D], ro[D];
    auto load = [&](int i, int step) {
        const int64_t s = min(step, end - 1);
        __builtin_memcpy(rv[i], __builtin_assume_aligned(vals + s * (256 * CT), 4 * CT), 4 * CT);
        uint32_t four = 0;
        __builtin_memcpy(&four, __builtin_assume_aligned(scales + s * (16 * SP), SP), SP);
        rs[i] = four;
        ro[i] = *reinterpret_cast<const uint32_t *>(offs + s * 64);
    };

    // ---- A: this thread's block of a slab, rows 4 rb and on, columns 8 kc and on (16 lanes
    // take four pieces of four blocks of rows, which a write finds on different banks) ----
    const T *A = static_cast<const T *>(p.A) + row0 * p.lda;
    const __amdgpu_buffer_rsrc_t a_rsrc = make_rsrc(A, VEC ? (uint32_t)(((rows - 1) * p.lda + p.k) * 2) : 0u);
    const int rb = ((tid >> 2) & 3) + 4 * ((tid >> 5) % MT), kc0 = (tid & 3) + 4 * ((tid >> 4) & 1) + 8 * (tid / (2 * BM));
    constexpr int KB = mx4_wide_columns(MT) / NB / 8;     // pieces of 8 columns from one block of a thread to its next
    u32x4 ra[AD][NB][4];
    uint32_t a_off[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
        a_off[r] = 4 * rb + r < rows ? (uint32_t)((4 * rb + r) * p.lda * 2) + kc0 * 16 : OOB;
    // (columns past the chunk's are no group's; past the last row's end they read zeros.
    // Inlined by order: as a call, single values kept ra in memory, 32 x 4096 x 4096 at
    // 16:32 off 16 bytes 110 us, so 34)
    auto load_a = [&](int d, int s0) __attribute__((always_inline)) {
        const int64_t base = mx4_chunk_base(p, min(s0, end));
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if constexpr (VEC) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    ra[d][b][r] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                        a_rsrc, (int)a_off[r], (int)(base * 2) + b * KB * 16, 0));
            } else {
                const int64_t c0 = base + (kc0 + b * KB) * 8;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t two[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int64_t c = c0 + 2 * j + h;
                            two[h] = c < p.k && 4 * rb + r < rows
                                         ? __builtin_bit_cast(uint16_t, A[(4 * rb + r) * p.lda + c]) : 0u;
                        }
                        ra[d][b][r][j] = two[0] | two[1] << 16;
                    }
            }
        }
    };
    auto swizzle = [](int c) { return (c ^ (c >> 3)) & SWZ; };
    auto store_a = [&](int d, int slot) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                u32x2 out[4];
                transpose_4x4(ra[d][b], half, out);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = (kc0 + b * KB) * 8 + 4 * half + j;
                    *reinterpret_cast<u32x2 *>(lds + slot * SLOT + c * PITCH + (((rb >> 2) ^ swizzle(c)) << 5) +
                                               8 * (rb & 3)) = out[j];
                }
            }
    };
    // NaN in the places this thread's stores will fill
    auto poison_a = [&](int slot) {
#pragma unroll
        for (int i = 0; i < NB * 8; ++i) {
            const int c = (kc0 + i / 8 * KB) * 8 + i % 8;
            *reinterpret_cast<u32x2 *>(lds + slot * SLOT + c * PITCH + (((rb >> 2) ^ swizzle(c)) << 5) + 8 * (rb & 3)) =
                u32x2{~0u, ~0u};
        }
    };

    f32x4 acc[CT][MT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8 *)(lds_void *)lds;
    auto compute = [&](int i, int step, int64_t c0, int slot) {
        if (step >= end) return;
        const int delta = (int)(mx4_base(p, step) - c0);
        uint32_t at[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int c = delta + (int)((x == 0 ? ro[i] & 0xffffu : ro[i] >> 16) >> 1);
            at[x] = lds0 + (uint32_t)(slot * SLOT + c * PITCH + (swizzle(c) << 5) + 8 * (lane & 3));
        }
        s16x8 a[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            s16x4 v[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds_u8 *)(uintptr_t)(at[x] ^ (t << 5)));
            a[t] = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
        mx4_pad<MT>(p, step, grp, a);
#pragma unroll
        for (int c = 0; c < CT; ++c) mx4_group<T, MT>(a, rv[i][c], mx4_scale_at(rs[i], c), acc[c]);
    };

    load_a(0, first);
#pragma unroll
    for (int i = 0; i < D; ++i) load(i, first + wk + i * WK);
    load_a(1, first + CHUNK);
    // a chunk: its slab, which has been on its way for AD chunks, into the other slot
    // (whose readers were through at the last barrier), the next one asked for; then D
    // groups a wave
    auto chunk = [&](int d, int s0, int slot) {
        store_a(d, slot);
        lds_sync();
        if constexpr (NMSPMM_POISON_LDS) poison_a(slot ^ 1);    // (free, as above)
        const int64_t c0 = mx4_chunk_base(p, s0);
#pragma unroll
        for (int i = 0; i < D; ++i) {
            compute(i, s0 + wk + i * WK, c0, slot);
            load(i, s0 + CHUNK + wk + i * WK);
        }
        load_a(d, s0 + AD * CHUNK);     // (last: a wait for the weight's loads is none for these)
    };
    for (int s0 = first; s0 < end; s0 += 2 * CHUNK) {
        chunk(0, s0, 0);
        if (s0 + CHUNK >= end) break;
        chunk(1, s0 + CHUNK, 1);
    }
    mx4_finish<T, MT, CT, WC>(p, reinterpret_cast<float *>(lds), acc, row0, col0, rows, split, Mx4First{});
}

}  // namespace nmspmm

#endif
