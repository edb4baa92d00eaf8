// The product with a weight in 4 bits (nmspmm_mx4_*): rounding to 4 bits,
// layout of the packed weight, the kernel for any shape, and the dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>

#include "nmspmm_half.h"
#include "nmspmm_internal.h"
#include "nmspmm_fp4.h"
#include "nmspmm_mx4.h"
#include "nmspmm_workspace.h"

namespace nmspmm {
namespace {

bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// ---- rounding to 4 bits ------------------------------------------------------

// One column's group of 32 rows a thread, so that a wave reads rows in whole
// lines; the rows are read twice, the second time from L2.
template <class S>
__global__ __launch_bounds__(256) void nm_mx4_quantize_kernel(const S *Bc, int64_t w, int64_t n, uint8_t *codes,
                                                              uint8_t *scales)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    for (int64_t g = blockIdx.y; g * 32 < w; g += gridDim.y) {
        const S *x = Bc + g * 32 * n + j;
        const int held = (int)min<int64_t>(32, w - g * 32);
        uint32_t top = 0;
        for (int u = 0; u < held; ++u) top = max(top, __builtin_bit_cast(uint32_t, to_f32(x[u * n])) & 0x7fffffffu);
        const uint32_t s = mx4_scale_of(top);
        scales[g * n + j] = (uint8_t)s;
        for (int u0 = 0; u0 < held; u0 += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = u0 + i < held ? to_f32(x[(u0 + i) * n]) : 0.f;
            const uint32_t c = mx4_codes(v, s);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (u0 + i < held) codes[(g * 32 + u0 + i) * n + j] = (uint8_t)(c >> (4 * i) & 15);
        }
    }
}

// ---- the packed weight -----------------------------------------------------
//
// Two compressed rows' codes a byte, row-major; the scales; the offsets (none
// where N = M: row r of a window is its r-th).
struct Mx4Layout {
    int64_t w, q, groups;
    int64_t scales_at, offs_at, bytes;
};

Mx4Layout mx4_layout(int64_t k, int64_t n, int N, int M, int V)
{
    Mx4Layout l{};
    l.w = k / M * N;
    l.q = n / V;
    l.groups = (l.w + 31) / 32;
    l.scales_at = round_up((l.w + 1) / 2 * n, 256);
    l.offs_at = round_up(l.scales_at + l.groups * n, 256);
    l.bytes = l.offs_at + (N == M ? 0 : l.w * l.q);
    return l;
}

__global__ __launch_bounds__(256) void nm_mx4_pack_raw_kernel(const uint8_t *codes, const uint8_t *scales,
                                                              const uint8_t *idx, uint8_t *out, Mx4Layout l, int64_t n,
                                                              int M)
{
    const int64_t stride = (int64_t)gridDim.x * 256, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t e = t; e < (l.w + 1) / 2 * n; e += stride) {
        const int64_t u = e / n * 2, j = e % n;
        const uint32_t hi = u + 1 < l.w ? codes[(u + 1) * n + j] & 15u : 0u;
        out[e] = (uint8_t)((codes[u * n + j] & 15u) | hi << 4);
    }
    for (int64_t e = t; e < l.groups * n; e += stride) out[l.scales_at + e] = scales[e];
    for (int64_t e = t; e < l.bytes - l.offs_at; e += stride) out[l.offs_at + e] = (uint8_t)(idx[e] < M ? idx[e] : M - 1);
}

// ---- any shape -------------------------------------------------------------

struct Mx4GeneralArgs {
    const void *A;
    const unsigned char *packed;
    Mx4Layout l;
    int64_t lda, m, n;
    int N, M, V;
    HalfEpilogue epi;
};

constexpr int MG_ROWS = 8;

// Any shape: a thread owns one column and MG_ROWS rows of C and walks the
// compressed rows; bound by the loads of A, one value per multiply-add.
template <class T, class O>
__global__ __launch_bounds__(256) void nm_mx4_general_kernel(Mx4GeneralArgs p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.n) return;
    const T *A = static_cast<const T *>(p.A);
    const unsigned char *scales = p.packed + p.l.scales_at;
    const unsigned char *offs = p.N == p.M ? nullptr : p.packed + p.l.offs_at + j / p.V;
    for (int64_t i0 = (int64_t)blockIdx.y * MG_ROWS; i0 < p.m; i0 += (int64_t)gridDim.y * MG_ROWS) {
        float sum[MG_ROWS] = {};
        int64_t window = 0;
        for (int64_t u = 0, r = 0; u < p.l.w; ++u) {
            const uint32_t code = p.packed[u / 2 * p.n + j] >> (u % 2 * 4) & 15u;
            const float s = mx4_scale<0>(scales[u / 32 * p.n + j]);
            const float b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0)[0];
            const T *a = A + i0 * p.lda + window + (offs ? offs[u * p.l.q] : r);
#pragma unroll
            for (int i = 0; i < MG_ROWS; ++i)
                if (i0 + i < p.m) sum[i] = fmaf(to_f32(a[i * p.lda]), b, sum[i]);
            if (++r == p.N) {
                r = 0;
                window += p.M;
            }
        }
#pragma unroll
        for (int i = 0; i < MG_ROWS; ++i)
            if (i0 + i < p.m) half_store<O>(p.epi, i0 + i, j, sum[i]);
    }
}

template <class T>
hipError_t launch_general(const Mx4GeneralArgs &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.n + 255) / 256),
                    (unsigned)std::min<int64_t>(65535, (p.m + MG_ROWS - 1) / MG_ROWS));
    if (p.epi.f32) hipLaunchKernelGGL((nm_mx4_general_kernel<T, float>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((nm_mx4_general_kernel<T, T>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

nmspmm_status_t check_weight(const nmspmm_mx4_weight_t *w, int64_t m)
{
    if (!w || !shape_ok(m, w->n, w->k, w->N, w->M, w->V)) return NMSPMM_ERR_INVALID_ARG;
    // a launch takes fewer than 2^32 threads, one a column
    if (!sizes_fit(m, w->n, w->k) || w->n >= ((int64_t)1 << 31) - 255) return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" int64_t nmspmm_mx4_bytes(int64_t k, int64_t n, int N, int M, int V)
{
    if (!shape_ok(0, n, k, N, M, V) || !sizes_fit(1, n, k)) return -1;
    if (k == 0 || n == 0) return 0;
    return mx4_layout(k, n, N, M, V).bytes;
}

extern "C" nmspmm_status_t nmspmm_mx4_quantize(const void *Bc, nmspmm_dtype_t bc_dtype, int64_t w, int64_t n,
                                               uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    if (w < 0 || n < 0 || !dtype_ok(bc_dtype)) return NMSPMM_ERR_INVALID_ARG;
    if (w == 0 || n == 0) return NMSPMM_OK;
    if (!Bc || !codes || !scales) return NMSPMM_ERR_INVALID_ARG;
    if (!aligned_to(Bc, dtype_bytes(bc_dtype)) || !sizes_fit(1, n, w) || w >= ((int64_t)1 << 31) - 255 ||
        n >= ((int64_t)1 << 31) - 255)
        return NMSPMM_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((n + 255) / 256), (unsigned)std::min<int64_t>(65535, (w + 31) / 32));
    if (bc_dtype == NMSPMM_F32)
        hipLaunchKernelGGL((nm_mx4_quantize_kernel<float>), grid, dim3(256), 0, stream, static_cast<const float *>(Bc),
                           w, n, codes, scales);
    else if (bc_dtype == NMSPMM_BF16)
        hipLaunchKernelGGL((nm_mx4_quantize_kernel<bf16_t>), grid, dim3(256), 0, stream,
                           static_cast<const bf16_t *>(Bc), w, n, codes, scales);
    else
        hipLaunchKernelGGL((nm_mx4_quantize_kernel<f16_t>), grid, dim3(256), 0, stream, static_cast<const f16_t *>(Bc),
                           w, n, codes, scales);
    return hipGetLastError() == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" nmspmm_status_t nmspmm_mx4_pack(const uint8_t *codes, const uint8_t *scales, const uint8_t *idx,
                                           const nmspmm_mx4_weight_t *weight, hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, 0);
    if (st != NMSPMM_OK) return st;
    const nmspmm_mx4_weight_t &w = *weight;
    if (w.k == 0 || w.n == 0) return NMSPMM_OK;
    if (!codes || !scales || (!idx && w.N != w.M) || !w.packed) return NMSPMM_ERR_INVALID_ARG;
    if (!aligned_to(w.packed, 256)) return NMSPMM_ERR_UNSUPPORTED;
    const Mx4Layout l = mx4_layout(w.k, w.n, w.N, w.M, w.V);
    const dim3 grid((unsigned)std::min<int64_t>(8192, (l.w * w.n + 511) / 512));
    hipLaunchKernelGGL(nm_mx4_pack_raw_kernel, grid, dim3(256), 0, stream, codes, scales, idx,
                       static_cast<uint8_t *>(const_cast<void *>(w.packed)), l, w.n, w.M);
    return hipGetLastError() == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" int64_t nmspmm_mx4_workspace_bytes(int64_t m, const nmspmm_mx4_weight_t *weight)
{
    return check_weight(weight, m) == NMSPMM_OK ? 0 : -1;
}

extern "C" const char *nmspmm_mx4_kernel_name(int64_t m, const nmspmm_mx4_weight_t *weight, int with_workspace)
{
    if (check_weight(weight, m) != NMSPMM_OK) return "invalid";
    if (m == 0 || weight->n == 0) return "none";
    (void)with_workspace;
    return "nm_mx4_general_kernel";
}

extern "C" nmspmm_status_t nmspmm_mx4_run(const void *A, int64_t lda, nmspmm_dtype_t a_dtype,
                                          const nmspmm_mx4_weight_t *weight, void *C, int64_t ldc,
                                          nmspmm_dtype_t c_dtype, int64_t m, float alpha, const float *bias,
                                          nmspmm_half_act_t act, const void *mul, int64_t ld_mul, const void *residual,
                                          int64_t ld_residual, void *workspace, size_t workspace_bytes,
                                          hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, m);
    if (st != NMSPMM_OK) return st;
    const nmspmm_mx4_weight_t &w = *weight;
    if ((a_dtype != NMSPMM_BF16 && a_dtype != NMSPMM_F16) || (c_dtype != NMSPMM_F32 && c_dtype != a_dtype) ||
        act < NMSPMM_HALF_ACT_NONE || act > NMSPMM_HALF_ACT_SILU)
        return NMSPMM_ERR_INVALID_ARG;
    if (m == 0 || w.n == 0) return NMSPMM_OK;
    if (!C || (w.k > 0 && (!A || !w.packed))) return NMSPMM_ERR_INVALID_ARG;
    if (m > 1 && (lda < w.k || ldc < w.n || (mul && ld_mul < w.n) || (residual && ld_residual < w.n)))
        return NMSPMM_ERR_INVALID_ARG;
    const int cs = dtype_bytes(c_dtype);
    if (!aligned_to(A, 2) || !aligned_to(w.packed, 256) || !aligned_to(C, cs) || !aligned_to(bias, 4) ||
        !aligned_to(mul, cs) || !aligned_to(residual, cs) || !aligned_to(workspace, 256))
        return NMSPMM_ERR_UNSUPPORTED;
    if (!sizes_fit(m, std::max({ldc, ld_mul, ld_residual}), lda)) return NMSPMM_ERR_UNSUPPORTED;
    (void)workspace_bytes;
    const Mx4Layout l = mx4_layout(w.k, w.n, w.N, w.M, w.V);
    const HalfEpilogue epi = {C, bias, mul, residual, ldc, ld_mul, ld_residual, alpha, act, c_dtype == NMSPMM_F32, false};
    const Mx4GeneralArgs p{A, static_cast<const unsigned char *>(w.packed), l, m == 1 ? w.k : lda, m, w.n, w.N, w.M,
                           w.V, epi};
    const hipError_t e = a_dtype == NMSPMM_BF16 ? launch_general<bf16_t>(p, stream) : launch_general<f16_t>(p, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}
