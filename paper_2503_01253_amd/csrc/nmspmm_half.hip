// The N:M sparse product in bf16 and fp16 (nmspmm_half_*): layout of the
// packed weight, the kernels for any shape, and the dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>

#include "nmspmm_half.h"
#include "nmspmm_internal.h"
#include "nmspmm_workspace.h"

namespace nmspmm {
namespace {

bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The plain layout: Bc in 16 bits, then (256-byte aligned) idx.
struct RawLayout {
    int64_t w, q, idx_at, bytes;
};

RawLayout raw_layout(int64_t k, int64_t n, int N, int M, int V)
{
    RawLayout r;
    r.w = k / M * N;
    r.q = n / V;
    r.idx_at = round_up(2 * r.w * n, 256);
    r.bytes = r.idx_at + r.w * r.q;
    return r;
}

template <class T, class S>
__global__ __launch_bounds__(256) void nm_half_pack_raw_kernel(const S *Bc, const uint8_t *idx, T *vals,
                                                               uint8_t *offs, int64_t count, int64_t icount, int M)
{
    const int64_t stride = (int64_t)gridDim.x * 256, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t e = t; e < count; e += stride) vals[e] = from_f32<T>(to_f32(Bc[e]));
    for (int64_t e = t; e < icount; e += stride) offs[e] = (uint8_t)(idx[e] < M ? idx[e] : M - 1);
}

struct RawArgs {
    const void *A, *vals;
    const uint8_t *offs;
    int64_t lda, m, n, w, q;
    int N, M, V;
    HalfEpilogue epi;
};

constexpr int HG_ROWS = 8;

// Any shape: a thread owns one column and HG_ROWS rows of C and walks the
// compressed rows; bound by the loads of A, one value per multiply-add.
template <class T, class O>
__global__ __launch_bounds__(256) void nm_half_general_kernel(RawArgs p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.n) return;
    const T *A = static_cast<const T *>(p.A), *vals = static_cast<const T *>(p.vals) + j;
    const uint8_t *offs = p.offs + j / p.V;
    for (int64_t i0 = (int64_t)blockIdx.y * HG_ROWS; i0 < p.m; i0 += (int64_t)gridDim.y * HG_ROWS) {
        float sum[HG_ROWS] = {};
        int64_t window = 0;
        for (int64_t u = 0, r = 0; u < p.w; ++u) {
            const float b = to_f32(vals[u * p.n]);
            const T *a = A + i0 * p.lda + window + offs[u * p.q];
#pragma unroll
            for (int i = 0; i < HG_ROWS; ++i)
                if (i0 + i < p.m) sum[i] = fmaf(to_f32(a[i * p.lda]), b, sum[i]);
            if (++r == p.N) {
                r = 0;
                window += p.M;
            }
        }
#pragma unroll
        for (int i = 0; i < HG_ROWS; ++i)
            if (i0 + i < p.m) half_store<O>(p.epi, i0 + i, j, sum[i]);
    }
}

template <class T>
hipError_t launch_general(const RawArgs &p, bool f32_out, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.n + 255) / 256),
                    (unsigned)std::min<int64_t>(65535, (p.m + HG_ROWS - 1) / HG_ROWS));
    if (f32_out) hipLaunchKernelGGL((nm_half_general_kernel<T, float>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((nm_half_general_kernel<T, T>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

nmspmm_status_t check_weight(const nmspmm_half_weight_t *w, int64_t m)
{
    if (!w || !shape_ok(m, w->n, w->k, w->N, w->M, w->V)) return NMSPMM_ERR_INVALID_ARG;
    if (w->dtype != NMSPMM_BF16 && w->dtype != NMSPMM_F16) return NMSPMM_ERR_INVALID_ARG;
    // a launch takes fewer than 2^32 threads, one a column
    if (!sizes_fit(m, w->n, w->k) || w->n >= (int64_t)1 << 31) return NMSPMM_ERR_UNSUPPORTED;
    return NMSPMM_OK;
}

template <class T>
hipError_t pack_raw(const void *Bc, nmspmm_dtype_t type, const uint8_t *idx, const nmspmm_half_weight_t &w,
                    hipStream_t stream)
{
    const RawLayout r = raw_layout(w.k, w.n, w.N, w.M, w.V);
    T *vals = static_cast<T *>(const_cast<void *>(w.packed));
    uint8_t *offs = static_cast<uint8_t *>(const_cast<void *>(w.packed)) + r.idx_at;
    const int64_t count = r.w * w.n, icount = r.w * r.q;
    const dim3 grid((unsigned)std::min<int64_t>(8192, (count + 255) / 256));
    if (type == NMSPMM_F32)
        hipLaunchKernelGGL((nm_half_pack_raw_kernel<T, float>), grid, dim3(256), 0, stream,
                           static_cast<const float *>(Bc), idx, vals, offs, count, icount, w.M);
    else
        hipLaunchKernelGGL((nm_half_pack_raw_kernel<T, T>), grid, dim3(256), 0, stream, static_cast<const T *>(Bc),
                           idx, vals, offs, count, icount, w.M);
    return hipGetLastError();
}

}  // namespace
}  // namespace nmspmm

using namespace nmspmm;

extern "C" int64_t nmspmm_half_bytes(int64_t k, int64_t n, int N, int M, int V)
{
    if (!shape_ok(0, n, k, N, M, V) || !sizes_fit(1, n, k)) return -1;
    if (k == 0 || n == 0) return 0;
    return raw_layout(k, n, N, M, V).bytes;
}

extern "C" nmspmm_status_t nmspmm_half_pack(const void *Bc, nmspmm_dtype_t bc_dtype, const uint8_t *idx,
                                            const nmspmm_half_weight_t *weight, hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, 0);
    if (st != NMSPMM_OK) return st;
    if (bc_dtype != NMSPMM_F32 && bc_dtype != weight->dtype) return NMSPMM_ERR_INVALID_ARG;
    if (weight->k == 0 || weight->n == 0) return NMSPMM_OK;
    if (!Bc || !idx || !weight->packed) return NMSPMM_ERR_INVALID_ARG;
    if (!aligned_to(Bc, dtype_bytes(bc_dtype)) || !aligned_to(weight->packed, 256)) return NMSPMM_ERR_UNSUPPORTED;
    const hipError_t e = weight->dtype == NMSPMM_BF16 ? pack_raw<bf16_t>(Bc, bc_dtype, idx, *weight, stream)
                                                      : pack_raw<f16_t>(Bc, bc_dtype, idx, *weight, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}

extern "C" int64_t nmspmm_half_workspace_bytes(int64_t m, const nmspmm_half_weight_t *weight)
{
    return check_weight(weight, m) == NMSPMM_OK ? 0 : -1;
}

extern "C" const char *nmspmm_half_kernel_name(int64_t m, const nmspmm_half_weight_t *weight, int)
{
    if (check_weight(weight, m) != NMSPMM_OK) return "invalid";
    if (m == 0 || weight->n == 0) return "none";
    return "nm_half_general_kernel";
}

extern "C" nmspmm_status_t nmspmm_half_run(const void *A, int64_t lda, const nmspmm_half_weight_t *weight, void *C,
                                           int64_t ldc, nmspmm_dtype_t c_dtype, int64_t m, float alpha,
                                           const float *bias, nmspmm_half_act_t act, const void *mul, int64_t ld_mul,
                                           const void *residual, int64_t ld_residual, void *workspace,
                                           size_t workspace_bytes, hipStream_t stream)
{
    const nmspmm_status_t st = check_weight(weight, m);
    if (st != NMSPMM_OK) return st;
    const nmspmm_half_weight_t &w = *weight;
    if ((c_dtype != NMSPMM_F32 && c_dtype != w.dtype) || act < NMSPMM_HALF_ACT_NONE || act > NMSPMM_HALF_ACT_SILU)
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
    const RawLayout r = raw_layout(w.k, w.n, w.N, w.M, w.V);
    RawArgs p{};
    p.A = A;
    p.vals = w.packed;
    p.offs = static_cast<const uint8_t *>(w.packed) + r.idx_at;
    p.lda = lda;
    p.m = m;
    p.n = w.n;
    p.w = r.w;
    p.q = r.q;
    p.N = w.N;
    p.M = w.M;
    p.V = w.V;
    p.epi = {C, bias, mul, residual, ldc, ld_mul, ld_residual, alpha, act};
    const hipError_t e = w.dtype == NMSPMM_BF16 ? launch_general<bf16_t>(p, c_dtype == NMSPMM_F32, stream)
                                                : launch_general<f16_t>(p, c_dtype == NMSPMM_F32, stream);
    return e == hipSuccess ? NMSPMM_OK : NMSPMM_ERR_HIP;
}
