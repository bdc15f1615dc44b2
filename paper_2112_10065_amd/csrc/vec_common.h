// Device helpers shared by the memory-bound kernels (group norm, optimizer, log-probabilities): vectors of fp32 or
// bf16 elements, their conversion, reductions inside a wavefront; and the checks of their entry points.
#pragma once
#include "../../include/dp.h"
#include <hip/hip_runtime.h>
#include <stdint.h>

void dp_set_error(const char *fmt, ...);   // dp_api.hip

namespace {

typedef unsigned short bf16_t;

template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }   // nearest even

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline dp_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return DP_OK;
    dp_set_error("%s launch: %s", what, hipGetErrorString(e));
    return DP_ERR_HIP;
}

}  // namespace
