// Shared by the units of the 16-bit product: the epilogue (device code).
#ifndef NMSPMM_HALF_H
#define NMSPMM_HALF_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nmspmm_dtype.h"
#include "nmspmm_serve.h"

namespace nmspmm {

// C[i][j] = act(alpha * sum + bias[j]) * mul[i][j] + residual[i][j], in fp32,
// rounded once.  mul and residual have C's type.
struct HalfEpilogue {
    void *C;
    const float *bias;
    const void *mul, *residual;
    int64_t ldc, ld_mul, ld_residual;
    float alpha;
    int act;
    bool f32;               // C, mul and residual are fp32
    bool vec;               // every row of every operand starts on 16 bytes
};

// e^x, x <= 0: a power of 2 whose exponent's rounding, which __expf leaves in
// (30 steps of the result at x = -67), is put right.  (expf: 2048 x 4096 x 11008
// with SiLU and a factor 120 us; so, and the quotient by a reciprocal, 114, as
// with __expf.)
__device__ __forceinline__ float half_exp(float x)
{
    constexpr float LOG2E = 1.44269502f, LOG2E_REST = 1.92596299e-8f;
    const float p = x * LOG2E, rest = fmaf(x, LOG2E_REST, fmaf(x, LOG2E, -p));
    const float t = __builtin_amdgcn_exp2f(p);
    return fmaf(t, rest * 0.693147181f, t);
}

__device__ __forceinline__ float half_act(float y, int act)
{
    if (act == NMSPMM_HALF_ACT_RELU) return y < 0.f ? 0.f : y;      // NaN stays NaN
    // erfc, not 1 + erf, of which nothing is left below y = -5.5
    if (act == NMSPMM_HALF_ACT_GELU) return 0.5f * y * erfcf(y * -0.70710678118f);
    if (act == NMSPMM_HALF_ACT_SILU) {
        // of -|y|: no overflow; below -104 it is 0 (and an infinity's is not NaN)
        const float t = half_exp(fmaxf(-fabsf(y), -104.f)), d = 1.f + t;
        const float r = __builtin_amdgcn_rcpf(d);               // and a step of Newton's: d is 1 to 2
        return y * ((y < 0.f ? t : 1.f) * fmaf(r, fmaf(-d, r, 1.f), r));
    }
    return y;
}

template <class O>
__device__ __forceinline__ void half_store(const HalfEpilogue &e, int64_t i, int64_t j, float sum)
{
    float y = e.alpha * sum;
    if (e.bias) y += e.bias[j];
    y = half_act(y, e.act);
    if (e.mul) y *= to_f32(static_cast<const O *>(e.mul)[i * e.ld_mul + j]);
    if (e.residual) y += to_f32(static_cast<const O *>(e.residual)[i * e.ld_residual + j]);
    static_cast<O *>(e.C)[i * e.ldc + j] = from_f32<O>(y);
}

// Eight columns of row i from column j on, all inside C.  `ahead`: where what
// mul (or, without a mul, residual) holds there has been fetched to, or null.
template <class O>
__device__ __forceinline__ void half_store8(const HalfEpilogue &e, int64_t i, int64_t j, float (&y)[8],
                                            const O *ahead = nullptr)
{
    float z[8];
    if (!e.vec) {
#pragma unroll 1
        for (int x = 0; x < 8; ++x) {
            float v = y[0];     // (a dynamic index would put y into memory)
#pragma unroll
            for (int s = 1; s < 8; ++s) v = x == s ? y[s] : v;
            half_store<O>(e, i, j + x, v);
        }
        return;
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) y[x] *= e.alpha;
    if (e.bias) {
        load_row<8, true>(e.bias + j, 8, z);
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] += z[x];
    }
    if (e.act == NMSPMM_HALF_ACT_RELU) {
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] = half_act(y[x], NMSPMM_HALF_ACT_RELU);
    } else if (e.act == NMSPMM_HALF_ACT_GELU) {
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] = half_act(y[x], NMSPMM_HALF_ACT_GELU);
    } else if (e.act == NMSPMM_HALF_ACT_SILU) {
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] = half_act(y[x], NMSPMM_HALF_ACT_SILU);
    }
    if (e.mul) {
        load_row<8, true>(ahead ? ahead : static_cast<const O *>(e.mul) + i * e.ld_mul + j, 8, z);
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] *= z[x];
    }
    if (e.residual) {
        load_row<8, true>(ahead && !e.mul ? ahead : static_cast<const O *>(e.residual) + i * e.ld_residual + j, 8, z);
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] += z[x];
    }
    store_row<8, true>(static_cast<O *>(e.C) + i * e.ldc + j, 8, y);
}

}  // namespace nmspmm

#endif
