// Element types of the 16-bit operators: conversions to and from fp32 (device
// code) and the sizes of nmspmm_dtype_t.
#ifndef NMSPMM_DTYPE_H
#define NMSPMM_DTYPE_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nmspmm_serve.h"

namespace nmspmm {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline bool dtype_ok(nmspmm_dtype_t t) { return t == NMSPMM_F32 || t == NMSPMM_BF16 || t == NMSPMM_F16; }
inline int dtype_bytes(nmspmm_dtype_t t) { return t == NMSPMM_F32 ? 4 : 2; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(f16_t x) { return (float)x; }
__device__ __forceinline__ float to_f32(bf16_t x)
{
    return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, x) << 16);
}

// Rounds to nearest, ties to even.
template <class T>
__device__ __forceinline__ T from_f32(float x)
{
    return (T)x;
}

// N consecutive elements at p as fp32: one 16- or 8-byte load each where VEC,
// else element by element, the first `valid` of them (zeros after).
template <int N, bool VEC, class T>
__device__ __forceinline__ void load_row(const T *p, int valid, float (&x)[N])
{
    if constexpr (VEC) {
        T v[N];
        if (valid >= N) {
            __builtin_memcpy(v, __builtin_assume_aligned(p, sizeof(T) * N < 16 ? sizeof(T) * N : 16), sizeof v);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = to_f32(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < valid ? to_f32(p[i]) : 0.f;
    }
}

// The same the other way round.
template <int N, bool VEC, class T>
__device__ __forceinline__ void store_row(T *p, int valid, const float (&x)[N])
{
    if constexpr (VEC) {
        if (valid >= N) {
            T v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = from_f32<T>(x[i]);
            __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T) * N < 16 ? sizeof(T) * N : 16), v, sizeof v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < valid) p[i] = from_f32<T>(x[i]);
    }
}

}  // namespace nmspmm

#endif
