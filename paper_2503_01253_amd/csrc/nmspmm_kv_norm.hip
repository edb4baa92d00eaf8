// New tokens into a paged cache with norms of the heads and rotary positions:
// nmspmm_kv_append_norm (a cache of 16- or 32-bit values) and nmspmm_kv4_append
// (one of 4 bits).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

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
    int32_t heads, rows, dim, rot, interleaved, log_team;
    float eps;
};

constexpr int AN_NT = 256, AN_NW = AN_NT / 64;

// What a row is combined with: a lane's eight dimensions, and those that turn
// with them (`with`), their norm's weights and the angles.
struct Piece {
    float x[8], with[8], w[8], w_with[8], c[8], s[8];   // s with the sign of with's term
};

// y = norm, then rotation, of a lane's piece.  F: the type to compute in.
template <class F>
__device__ __forceinline__ void norm_and_turn(const Piece &a, F (&y)[8], bool norm, bool rotate, int log_team, int dim,
                                              float eps)
{
    F inv = 1;
    if (norm) {     // the sum in fp64: squares of large fp32 values stay finite
        double sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)a.x[i], (double)a.x[i], sum);
        for (int step = 1; step < 1 << log_team; step *= 2) sum += __shfl_xor(sum, step);
        inv = (F)(1 / sqrt(sum / dim + (double)eps));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        F own = a.x[i], with = a.with[i];
        if (norm) {
            own *= inv * (F)a.w[i];
            with *= inv * (F)a.w_with[i];
        }
        if (!rotate) y[i] = own;
        else if constexpr (__is_same(F, double)) y[i] = fma(own, (double)a.c[i], with * (double)a.s[i]);
        else y[i] = fmaf(own, a.c[i], with * a.s[i]);
    }
}

// A wave takes one row (a key, value or query head) of 64 >> log_team tokens: a
// team of 1 << log_team lanes a token, eight dimensions a lane, so that a norm's
// sum and a group's largest magnitude are found between lanes.  A dimension's
// partner in the rotation is loaded beside it (from the same lines).  VEC: rows
// and angles in whole 16-byte pieces.  C: the cache's type, or Fp4.
template <class T, class C, bool VEC>
__global__ __launch_bounds__(AN_NT) void nm_append_norm_kernel(NormArgs p)
{
    constexpr bool FP4 = __is_same(C, Fp4);
    const int lane = threadIdx.x & 63, sub = lane & ((1 << p.log_team) - 1);
    const int row = blockIdx.y * AN_NW + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= p.rows) return;
    const int64_t t = (int64_t)blockIdx.x * (64 >> p.log_team) + (lane >> p.log_team);
    bool there = t < p.tokens;
    const bool is_k = row < p.heads, is_v = !is_k && row < 2 * p.heads;
    const int head = is_k ? row : is_v ? row - p.heads : row - 2 * p.heads;
    const float *weight = is_k ? p.k_norm : is_v ? nullptr : p.q_norm;
    const int d0 = sub * 8, valid = p.dim - d0 < 0 ? 0 : p.dim - d0 < 8 ? p.dim - d0 : 8;
    const int half = p.rot / 2;
    const bool rotate = !is_v && p.rot > 0;

    Piece a;
    const int64_t pos = there ? p.pos[t] : -1, seq = there ? p.seq[t] : -1;
    const T *src = is_k ? static_cast<const T *>(p.k_new) + t * p.kn[0] + head * p.kn[1]
                 : is_v ? static_cast<const T *>(p.v_new) + t * p.vn[0] + head * p.vn[1]
                        : static_cast<const T *>(p.q) + t * p.qn[0] + head * p.qn[1];
    load_row<8, VEC>(src + d0, there ? valid : 0, a.x);
    if (weight) load_row<8, VEC>(weight + d0, valid, a.w);
    // the partners: of a pair (d, d + half) in other lanes, of (2d, 2d + 1) in this one
    const bool apart = rotate && !p.interleaved;
    if (apart) {
        if constexpr (VEC) {
            const int at = d0 < half ? d0 + half : d0 < p.rot ? d0 - half : d0;
            load_row<8, true>(src + at, there ? valid : 0, a.with);
            if (weight) load_row<8, true>(weight + at, valid, a.w_with);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = d0 + i, at = d < half ? d + half : d < p.rot ? d - half : d;
                a.with[i] = there && i < valid ? to_f32(src[at]) : 0.f;
                a.w_with[i] = weight && i < valid ? weight[at] : 0.f;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a.with[i] = a.x[i ^ 1];
            if (weight) a.w_with[i] = a.w[i ^ 1];
        }
    }

    there = there && pos >= 0 && pos < p.table_positions && seq >= 0 && seq < p.sequences &&
            !(p.rot && pos >= p.positions);
    Place at{0, 0, false};
    if (there) at = place_of(p.c, p.c.table + seq * p.c.table_stride, (int)pos);
    there = there && at.held;

    if (rotate) {
        const int64_t angles = (there ? pos : 0) * half;
#pragma unroll
        for (int i = 0; i < 8; ++i) a.c[i] = 1.f, a.s[i] = 0.f;
        if constexpr (VEC) {
            if (there && d0 < p.rot) {
                if (apart) {
                    const int e = d0 < half ? d0 : d0 - half;
                    load_row<8, true>(p.cos + angles + e, 8, a.c);
                    load_row<8, true>(p.sin + angles + e, 8, a.s);
                } else {
                    float c[4], s[4];
                    load_row<4, true>(p.cos + angles + d0 / 2, 4, c);
                    load_row<4, true>(p.sin + angles + d0 / 2, 4, s);
#pragma unroll
                    for (int i = 0; i < 8; ++i) a.c[i] = c[i / 2], a.s[i] = s[i / 2];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = d0 + i;
                if (there && d < p.rot) {
                    const int e = apart ? (d < half ? d : d - half) : d / 2;
                    a.c[i] = p.cos[angles + e];
                    a.s[i] = p.sin[angles + e];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (apart ? d0 + i < half : i % 2 == 0) a.s[i] = -a.s[i];
    }

    float y[8];
    if (FP4 && is_k && (weight || rotate)) {
        double z[8];
        norm_and_turn<double>(a, z, weight != nullptr, rotate, p.log_team, p.dim, p.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = mx4_narrow(z[i]);
    } else {
        norm_and_turn<float>(a, y, weight != nullptr, rotate, p.log_team, p.dim, p.eps);
    }

    if (!is_k && !is_v) {
        if (there) store_row<8, VEC>(static_cast<T *>(p.q_out) + t * p.qo[0] + head * p.qo[1] + d0, valid, y);
        return;
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

template <class T, class C>
hipError_t launch_norm_to(const NormArgs &p, bool vec, hipStream_t stream)
{
    const int64_t per = 64 >> p.log_team;
    const dim3 grid((unsigned)((p.tokens + per - 1) / per), (unsigned)((p.rows + AN_NW - 1) / AN_NW));
    if (vec) hipLaunchKernelGGL((nm_append_norm_kernel<T, C, true>), grid, dim3(AN_NT), 0, stream, p);
    else hipLaunchKernelGGL((nm_append_norm_kernel<T, C, false>), grid, dim3(AN_NT), 0, stream, p);
    return hipGetLastError();
}

template <class T>
hipError_t launch_norm(const NormArgs &p, bool four, nmspmm_dtype_t cache, bool vec, hipStream_t stream)
{
    if (four) return launch_norm_to<T, Fp4>(p, vec, stream);
    if (cache == NMSPMM_F32) return launch_norm_to<T, float>(p, vec, stream);
    return cache == NMSPMM_BF16 ? launch_norm_to<T, bf16_t>(p, vec, stream) : launch_norm_to<T, f16_t>(p, vec, stream);
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
    // a launch takes fewer than 2^32 threads along x and 2^16 workgroups along y
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
    p.rows = (int)rows;
    p.dim = cache->dim;
    p.rot = n.rot;
    p.interleaved = n.interleaved != 0;
    p.eps = n.eps;
    for (p.log_team = 2; 8 << p.log_team < cache->dim;) ++p.log_team;
    const int es = dtype_bytes(n.dtype), cs = dtype_bytes(cache->dtype);
    const bool vec = cache->dim % 8 == 0 && (n.interleaved ? n.rot % 8 == 0 : n.rot % 16 == 0) &&
                     rows_aligned(n.k, n.ks, 2, cache->dim, es) && rows_aligned(n.v, n.vs, 2, cache->dim, es) &&
                     aligned_to(n.cos, 16) && aligned_to(n.sin, 16) && aligned_to(n.q_norm, 16) &&
                     aligned_to(n.k_norm, 16) &&
                     (n.q_heads == 0 || (rows_aligned(n.q, n.qs, 2, cache->dim, es) &&
                                         rows_aligned(n.q_out, n.qos, 2, cache->dim, es))) &&
                     (four || (rows_aligned(cache->k_pages, cache->k_stride, 3, cache->dim, cs) &&
                               rows_aligned(cache->v_pages, cache->v_stride, 3, cache->dim, cs)));
    const bool f = four != nullptr;
    const hipError_t e = n.dtype == NMSPMM_F32    ? launch_norm<float>(p, f, cache->dtype, vec, stream)
                         : n.dtype == NMSPMM_BF16 ? launch_norm<bf16_t>(p, f, cache->dtype, vec, stream)
                                                  : launch_norm<f16_t>(p, f, cache->dtype, vec, stream);
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
