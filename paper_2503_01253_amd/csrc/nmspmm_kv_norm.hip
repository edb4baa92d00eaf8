// New tokens into a paged cache with norms of the heads and rotary positions:
// nmspmm_kv_append_norm (a cache of 16- or 32-bit values) and nmspmm_kv4_append
// (one of 4 bits).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "nmspmm_kv4.h"
#include "nmspmm_kv_host.h"

namespace nmspmm {
namespace {

struct Fp4 {};      // in the place of a cache's element type

struct NormArgs {
    Pages c;
    Kv4Pages f;
    const void *k_new, *v_new, *q;
    void *k_pages, *v_pages, *q_out;
    int64_t kn[2], vn[2], qn[2], qo[2];
    const int32_t *seq, *pos;
    const float *cos, *sin, *q_norm, *k_norm;
    int64_t tokens, positions, sequences, table_positions;
    int64_t first_token;
    int32_t heads, q_heads, dim, rot, interleaved, log_team;
    int32_t slices[3];      // waves that share a group of tokens: for its keys, values and queries
    float eps;
    double inv_dim;
};

// How a row is read: value by value; in whole 16-byte pieces; and so also the
// pieces that turn with them, and the angles.
enum NormMode { AN_SINGLE, AN_ROWS, AN_WHOLE };

constexpr int AN_NT = 256, AN_NW = AN_NT / 64;

// The sum of x over a team of 1 << log_team lanes, in every one of them.
__device__ __forceinline__ double team_sum(double x, int log_team)
{
    auto dpp = [](double v, auto ctrl) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        constexpr int C = decltype(ctrl)::value;
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, C, 0xf, 0xf, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), C, 0xf, 0xf, false);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    x += dpp(x, std::integral_constant<int, 0xb1>{});                           // lane ^ 1
    x += dpp(x, std::integral_constant<int, 0x4e>{});                           // lane ^ 2
    if (log_team >= 3) x += dpp(x, std::integral_constant<int, 0x141>{});       // the other four of eight
    if (log_team >= 4) x += dpp(x, std::integral_constant<int, 0x140>{});       // the other eight of sixteen
    if (log_team >= 5) x += __shfl_xor(x, 16);
    if (log_team >= 6) x += __shfl_xor(x, 32);
    return x;
}

// 1 / sqrt(m) in fp64 from the instruction's estimate (23 bits) and `steps` of
// Newton's iteration, each of which doubles them.
template <int STEPS>
__device__ __forceinline__ double inverse_root(double m)
{
    const double first = __builtin_amdgcn_rsq(m);
    double y = first;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) y = fma(0.5 * y, fma(-m * y, y, 1.0), y);
    return m > 0 && m < __builtin_inf() ? y : first;
}

// A lane's eight dimensions of a row, and those that turn with them.
template <class T>
struct RowPiece {
    alignas(8 * sizeof(T) < 16 ? 8 * sizeof(T) : 16) T x[8], with[8];
};

// A wave takes one token and ROWS times 64 >> log_team heads of its keys, its
// values or its queries: a team of 1 << log_team lanes a head, eight dimensions a
// lane, so that a norm's sum and a group's largest magnitude are found between
// lanes.  The place and the angles are found once for all of them, and all heads
// are loaded before anything is waited for.  The dimensions that turn with a
// lane's come from another lane (WHOLE), or are loaded beside them.  C: the
// cache's type, or Fp4: then the keys are computed in fp64, where the weights'
// products with the angles are exact, and get the codes of the formula.
//
// Bound by memory, and for few tokens by the chain pos -> table -> store: 4001
// tokens of 48 rows of 128 (32 queries, 8 keys and values), both norms, rotation
// of all dimensions: fp32 into bf16 39 us, 4.6 TB/s; bf16 into bf16 29 us, 3.4
// TB/s; bf16 into 4 bits 34 us.  64 tokens take 4.5 us.  A wave with four tokens
// and one head of them took 50, 44 and 50 us, one that goes over many heads in a
// loop 44, 37 and 40 (it waits for its stores).
template <class T, class C, NormMode MODE, int ROWS>
__global__ __launch_bounds__(AN_NT) void nm_append_norm_kernel(NormArgs p)
{
    constexpr bool FP4 = __is_same(C, Fp4), VEC = MODE != AN_SINGLE, WHOLE = MODE == AN_WHOLE;
    const int lane = threadIdx.x & 63, sub = lane & ((1 << p.log_team) - 1);
    const uint32_t wave = blockIdx.x * AN_NW + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t per_group = p.slices[0] + p.slices[1] + p.slices[2], group = wave / per_group;
    int slice = (int)(wave - group * per_group);
    const bool is_k = slice < p.slices[0], is_v = !is_k && slice < p.slices[0] + p.slices[1], is_q = !is_k && !is_v;
    slice -= is_k ? 0 : is_v ? p.slices[0] : p.slices[0] + p.slices[1];
    const int per = 64 >> p.log_team, begin = slice * ROWS * per + (lane >> p.log_team), heads = is_q ? p.q_heads : p.heads;
    const int64_t t = p.first_token + group;
    if (t >= p.tokens) return;
    const int d0 = sub * 8, valid = p.dim - d0 < 0 ? 0 : p.dim - d0 < 8 ? p.dim - d0 : 8;
    const int half = p.rot / 2;
    const bool rotate = !is_v && p.rot > 0;
    const float *w = is_k ? p.k_norm : is_v ? nullptr : p.q_norm;
    // partners: of a pair (d, d + half) in other lanes, of (2d, 2d + 1) in this one
    const bool apart = rotate && !p.interleaved;
    // (lanes past the row read its start, and their values are not used)
    const int from = valid > 0 ? d0 : 0, other = !apart || from >= p.rot ? from : from < half ? from + half : from - half;

    auto partner = [&](int d) { return d < half ? d + half : d < p.rot ? d - half : d; };
    const T *src = is_k ? static_cast<const T *>(p.k_new) + t * p.kn[0]
                 : is_v ? static_cast<const T *>(p.v_new) + t * p.vn[0]
                        : static_cast<const T *>(p.q) + t * p.qn[0];
    const int64_t head_stride = is_k ? p.kn[1] : is_v ? p.vn[1] : p.qn[1];
    RowPiece<T> rows[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        RowPiece<T> &a = rows[r];
        const T *row = src + (begin + r * per < heads ? begin + r * per : heads - 1) * head_stride;
        if constexpr (VEC) __builtin_memcpy(a.x, __builtin_assume_aligned(row + from, 16), sizeof(a.x));
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) a.x[i] = i < valid ? row[d0 + i] : T(0);
        if constexpr (!WHOLE)
#pragma unroll
            for (int i = 0; i < 8; ++i) a.with[i] = apart && i < valid ? row[partner(d0 + i)] : T(0);
    }
    const int64_t pos = p.pos[t], seq = p.seq[t];
    if (pos < 0 || pos >= p.table_positions || seq < 0 || seq >= p.sequences || (p.rot && pos >= p.positions)) return;
    const Place at = place_of(p.c, p.c.table + seq * p.c.table_stride, (int)pos);
    if (!at.held) return;

    auto first = [&](int i) { return apart ? d0 + i < half : i % 2 == 0; };     // of its pair
    auto finish = [&](auto in) {
        using F = decltype(in);
        // y = x * f + with * g: the norm's weights times cos and sin; with and g are
        // zero where nothing turns (and g -0, which leaves x's sign if x is zero)
        F f[8], g[8];
        if (w || rotate) {
            float c[8], s[8], u[8], v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = u[i] = v[i] = 1.f, s[i] = 0.f;
            if (rotate && d0 < p.rot) {
                const int64_t angles = pos * half;
                if (WHOLE && apart) {
                    const int e = d0 < half ? d0 : d0 - half;
                    load_row<8, true>(p.cos + angles + e, 8, c);
                    load_row<8, true>(p.sin + angles + e, 8, s);
                } else if (WHOLE) {
                    float c4[4], s4[4];
                    load_row<4, true>(p.cos + angles + d0 / 2, 4, c4);
                    load_row<4, true>(p.sin + angles + d0 / 2, 4, s4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) c[i] = c4[i / 2], s[i] = s4[i / 2];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int d = d0 + i, e = apart ? (d < half ? d : d - half) : d / 2;
                        if (d < p.rot) c[i] = p.cos[angles + e], s[i] = p.sin[angles + e];
                    }
                }
            }
            if (w) {
                if (WHOLE) {
                    load_row<8, true>(w + from, 8, u);
                    load_row<8, true>(w + other, 8, v);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        u[i] = i < valid ? w[d0 + i] : 0.f;
                        v[i] = i < valid && apart ? w[partner(d0 + i)] : 0.f;
                    }
                }
                if (!apart)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = u[i ^ 1];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = (F)c[i] * (F)u[i];
                g[i] = rotate && d0 + i < p.rot ? (F)(first(i) ? -s[i] : s[i]) * (F)v[i] : F(-0.0);
            }
        }

#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int head = begin + r * per;
            const bool there = head < heads;
            RowPiece<T> &a = rows[r];
            if constexpr (WHOLE) {
                if (apart) {
                    int u[sizeof(a.x) / 4];
                    __builtin_memcpy(u, a.x, sizeof(a.x));
#pragma unroll
                    for (int &word : u) word = __builtin_amdgcn_ds_bpermute(4 * lane + (other - from) / 2, word);
                    __builtin_memcpy(a.with, u, sizeof(u));
                }
            }
            float y[8];
            if (!w && !rotate) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = to_f32(a.x[i]);
            } else {
                float with[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) with[i] = apart ? to_f32(a.with[i]) : to_f32(a.x[i ^ 1]);
                if (p.rot < p.dim)
#pragma unroll
                    for (int i = 0; i < 8; ++i) with[i] = d0 + i < p.rot ? with[i] : 0;
                double inv = 1;
                if (w) {
                    double mean = 0;    // in fp64: squares of large fp32 values stay finite
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const double x = to_f32(a.x[i]);
                        mean = fma(x, x, mean);
                    }
                    mean = team_sum(valid > 0 ? mean : 0, p.log_team) * p.inv_dim + (double)p.eps;
                    inv = inverse_root<__is_same(F, double) ? 2 : 1>(mean);
                }
                // (in fp64 too where fp32 does not hold the factor: rows of tiny or huge values;
                // by a team's own, so that a head's bits do not depend on its neighbours)
                const bool far = !(inv >= 0x1p-120 && inv <= 0x1p120);
                if (__is_same(F, double) || far) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const double z = inv * fma((double)to_f32(a.x[i]), (double)f[i], (double)with[i] * (double)g[i]);
                        y[i] = __is_same(F, double) ? mx4_narrow(z) : (float)z;
                    }
                } else if (!w) {        // as nmspmm_kv_append rounds
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        y[i] = turn_one(to_f32(a.x[i]), with[i], (float)f[i], (float)g[i], !first(i));
                } else {
                    const float inv32 = (float)inv;
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = fmaf(to_f32(a.x[i]) * inv32, (float)f[i], with[i] * inv32 * (float)g[i]);
                }
            }

            if (is_q) {
                if (there) store_row<8, VEC>(static_cast<T *>(p.q_out) + t * p.qo[0] + head * p.qo[1] + d0, valid, y);
                continue;
            }
            if constexpr (FP4) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i >= valid) y[i] = 0.f;
                    top = max(top, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);
                }
                top = max(top, (uint32_t)__shfl_xor((int)top, 1));      // the four lanes of a group
                top = max(top, (uint32_t)__shfl_xor((int)top, 2));
                const uint32_t scale = mx4_scale_of(top), codes = mx4_codes(y, scale);
                if (there && sub < 4 * p.f.l.G) {
                    unsigned char *b = p.f.block(at.page, head);
                    *reinterpret_cast<uint32_t *>(b + (is_k ? p.f.l.k_word(at.slot, sub) : p.f.l.v_word(at.slot, sub))) = codes;
                    if (sub % 4 == 0)
                        b[is_k ? p.f.l.k_scale(at.slot, sub / 4) : p.f.l.v_scale(at.slot, sub / 4)] = (unsigned char)scale;
                }
            } else if (there) {
                C *dst = is_k ? static_cast<C *>(p.k_pages) + at.page * p.c.ks[0] + at.slot * p.c.ks[1] + head * p.c.ks[2]
                              : static_cast<C *>(p.v_pages) + at.page * p.c.vs[0] + at.slot * p.c.vs[1] + head * p.c.vs[2];
                store_row<8, VEC>(dst + d0, valid, y);
            }
        }
    };
    if (FP4 && is_k) finish(0.0);
    else finish(0.f);
}

template <class T, class C, NormMode MODE, int ROWS>
hipError_t launch_norm_rows(NormArgs p, hipStream_t stream)
{
    const int rows = ROWS * (64 >> p.log_team);
    p.slices[0] = p.slices[1] = (p.heads + rows - 1) / rows;
    p.slices[2] = (p.q_heads + rows - 1) / rows;
    const int64_t slices = 2 * (int64_t)p.slices[0] + p.slices[2];
    // a grid takes fewer than 2^32 threads, and all but the last end with their waves: a
    // query that is turned in place is read once
    const int64_t most = ((int64_t)1 << 25) / slices / AN_NW * AN_NW;
    for (; p.first_token < p.tokens; p.first_token += most) {
        const int64_t groups = std::min(most, p.tokens - p.first_token);
        const dim3 grid((unsigned)((groups * slices + AN_NW - 1) / AN_NW));
        hipLaunchKernelGGL((nm_append_norm_kernel<T, C, MODE, ROWS>), grid, dim3(AN_NT), 0, stream, p);
    }
    return hipGetLastError();
}

template <class T, class C>
hipError_t launch_norm_to(const NormArgs &p, NormMode mode, hipStream_t stream)
{
    // two steps of heads a wave where that still fills the card (512 tokens of 48 rows of
    // 128 into 4 bits: 8.4 us with one, 9.0 with two; 4001 tokens: 41 and 35)
    const bool many = (p.tokens << p.log_team) / 64 * (2 * (int64_t)p.heads + p.q_heads) >= 8192;
    if (mode == AN_WHOLE)
        return many ? launch_norm_rows<T, C, AN_WHOLE, 2>(p, stream) : launch_norm_rows<T, C, AN_WHOLE, 1>(p, stream);
    if (mode == AN_ROWS)
        return many ? launch_norm_rows<T, C, AN_ROWS, 2>(p, stream) : launch_norm_rows<T, C, AN_ROWS, 1>(p, stream);
    return launch_norm_rows<T, C, AN_SINGLE, 1>(p, stream);
}

template <class T>
hipError_t launch_norm(const NormArgs &p, bool four, nmspmm_dtype_t cache, NormMode mode,
                       hipStream_t stream)
{
    if (four) return launch_norm_to<T, Fp4>(p, mode, stream);
    if (cache == NMSPMM_F32) return launch_norm_to<T, float>(p, mode, stream);
    return cache == NMSPMM_BF16 ? launch_norm_to<T, bf16_t>(p, mode, stream) : launch_norm_to<T, f16_t>(p, mode, stream);
}

// What the two entry points share.  cache: sizes and table; four: the 4-bit
// cache's pages, or null.
struct NewTokens {
    const void *k, *v, *q;
    void *q_out;
    const int64_t *ks, *vs, *qs, *qos;
    nmspmm_dtype_t dtype;
    int64_t tokens, positions, q_heads;
    const int32_t *seq, *pos;
    const float *cos, *sin, *q_norm, *k_norm;
    int rot, interleaved;
    float eps;
};

// After the cache's own checks; *done: nothing is left to do.
nmspmm_status_t check_new(const nmspmm_kv_cache_t *cache, const NewTokens &n, bool *done)
{
    *done = true;
    if (!dtype_ok(n.dtype) || n.tokens < 0 || n.positions < 0 || n.q_heads < 0 || n.rot < 0 || n.rot % 2 ||
        n.rot > cache->dim || !(n.eps >= 0.f))
        return NMSPMM_ERR_INVALID_ARG;
    if (n.tokens == 0) return NMSPMM_OK;
    *done = false;
    return NMSPMM_OK;
}

nmspmm_status_t check_new_pointers(const NewTokens &n)
{
    if (!n.k || !n.v || !n.ks || !n.vs || !n.seq || !n.pos) return NMSPMM_ERR_INVALID_ARG;
    if (n.rot > 0 && n.positions > 0 && (!n.cos || !n.sin)) return NMSPMM_ERR_INVALID_ARG;
    if (n.q_heads > 0 && (!n.q || !n.q_out || !n.qs || !n.qos)) return NMSPMM_ERR_INVALID_ARG;
    const int es = dtype_bytes(n.dtype);
    for (const void *x : {n.k, n.v, n.q, (const void *)n.q_out})
        if (!aligned_to(x, es)) return NMSPMM_ERR_UNSUPPORTED;
    for (const void *x : {(const void *)n.seq, (const void *)n.pos, (const void *)n.cos, (const void *)n.sin,
                          (const void *)n.q_norm, (const void *)n.k_norm})
        if (!aligned_to(x, 4)) return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

nmspmm_status_t append_new(const nmspmm_kv_cache_t *cache, const nmspmm_kv4_cache_t *four, const NewTokens &n,
                           hipStream_t stream)
{
    const int64_t rows = 2 * (int64_t)cache->heads + (n.q_heads > INT31 ? INT31 : n.q_heads);
    // the sizes of nmspmm_kv_append
    if (n.tokens >= (int64_t)1 << 24 || rows >= (int64_t)1 << 17 || n.positions > INT31) return NMSPMM_ERR_UNSUPPORTED;
    NormArgs p{};
    p.c = device_view(cache);
    if (four) p.f = kv4_view(four);
    p.k_new = n.k;
    p.v_new = n.v;
    p.q = n.q;
    p.k_pages = cache->k_pages;
    p.v_pages = cache->v_pages;
    p.q_out = n.q_out;
    for (int i = 0; i < 2; ++i) {
        p.kn[i] = n.ks[i];
        p.vn[i] = n.vs[i];
        p.qn[i] = n.q_heads ? n.qs[i] : 0;
        p.qo[i] = n.q_heads ? n.qos[i] : 0;
    }
    p.seq = n.seq;
    p.pos = n.pos;
    p.cos = n.cos;
    p.sin = n.sin;
    p.q_norm = n.q_norm;
    p.k_norm = n.k_norm;
    p.tokens = n.tokens;
    p.positions = n.positions;
    p.sequences = cache->sequences;
    p.table_positions = table_positions(cache);
    p.heads = cache->heads;
    p.q_heads = (int)n.q_heads;
    p.dim = cache->dim;
    p.rot = n.rot;
    p.interleaved = n.interleaved != 0;
    p.eps = n.eps;
    p.inv_dim = 1.0 / cache->dim;
    for (p.log_team = 2; 8 << p.log_team < cache->dim;) ++p.log_team;
    const int es = dtype_bytes(n.dtype), cs = dtype_bytes(cache->dtype);
    const bool whole = (n.interleaved ? n.rot % 8 == 0 : n.rot % 16 == 0) && aligned_to(n.cos, 16) && aligned_to(n.sin, 16);
    const bool vec = cache->dim % 8 == 0 && rows_aligned(n.k, n.ks, 2, cache->dim, es) &&
                     rows_aligned(n.v, n.vs, 2, cache->dim, es) && aligned_to(n.q_norm, 16) && aligned_to(n.k_norm, 16) &&
                     (n.q_heads == 0 || (rows_aligned(n.q, n.qs, 2, cache->dim, es) &&
                                         rows_aligned(n.q_out, n.qos, 2, cache->dim, es))) &&
                     (four || (rows_aligned(cache->k_pages, cache->k_stride, 3, cache->dim, cs) &&
                               rows_aligned(cache->v_pages, cache->v_stride, 3, cache->dim, cs)));
    const NormMode mode = !vec ? AN_SINGLE : whole ? AN_WHOLE : AN_ROWS;
    const bool f = four != nullptr;
    const hipError_t e = n.dtype == NMSPMM_F32    ? launch_norm<float>(p, f, cache->dtype, mode, stream)
                         : n.dtype == NMSPMM_BF16 ? launch_norm<bf16_t>(p, f, cache->dtype, mode, stream)
                                                  : launch_norm<f16_t>(p, f, cache->dtype, mode, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" nmspmm_status_t nmspmm_kv_append_norm(const nmspmm_kv_cache_t *cache, const void *k_new,
                                                 const int64_t *k_stride, const void *v_new, const int64_t *v_stride,
                                                 nmspmm_dtype_t dtype, int64_t tokens, const int32_t *seq,
                                                 const int32_t *pos, const float *cos, const float *sin,
                                                 int64_t positions, int rot, int interleaved, const float *q_norm,
                                                 const float *k_norm, float eps, const void *q,
                                                 const int64_t *q_stride, void *q_out, const int64_t *q_out_stride,
                                                 int64_t q_heads, hipStream_t stream)
{
    const NewTokens n{k_new, v_new, q, q_out, k_stride, v_stride, q_stride, q_out_stride, dtype, tokens, positions,
                      q_heads, seq, pos, cos, sin, q_norm, k_norm, rot, interleaved, eps};
    bool done;
    nmspmm_status_t st = check_cache(cache);
    if (st == NMSPMM_OK) st = check_new(cache, n, &done);
    if (st != NMSPMM_OK || done) return st;
    st = check_cache_pointers(cache);
    if (st == NMSPMM_OK) st = check_new_pointers(n);
    return st == NMSPMM_OK ? append_new(cache, nullptr, n, stream) : st;
}

extern "C" nmspmm_status_t nmspmm_kv4_append(const nmspmm_kv4_cache_t *cache, const void *k_new,
                                             const int64_t *k_stride, const void *v_new, const int64_t *v_stride,
                                             nmspmm_dtype_t dtype, int64_t tokens, const int32_t *seq,
                                             const int32_t *pos, const float *cos, const float *sin, int64_t positions,
                                             int rot, int interleaved, const float *q_norm, const float *k_norm,
                                             float eps, const void *q, const int64_t *q_stride, void *q_out,
                                             const int64_t *q_out_stride, int64_t q_heads, hipStream_t stream)
{
    const NewTokens n{k_new, v_new, q, q_out, k_stride, v_stride, q_stride, q_out_stride, dtype, tokens, positions,
                      q_heads, seq, pos, cos, sin, q_norm, k_norm, rot, interleaved, eps};
    nmspmm_status_t st = check_kv4(cache);
    if (st != NMSPMM_OK) return st;
    const nmspmm_kv_cache_t sizes = kv4_sizes(cache);
    bool done;
    st = check_new(&sizes, n, &done);
    if (st != NMSPMM_OK || done) return st;
    st = check_kv4_pointers(cache);
    if (st == NMSPMM_OK) st = check_new_pointers(n);
    return st == NMSPMM_OK ? append_new(&sizes, cache, n, stream) : st;
}
