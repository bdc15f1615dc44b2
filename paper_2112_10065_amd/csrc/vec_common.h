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

// A vector that is read or written once: past the caches, where it would push out lines that are still wanted, or dirty ones in the
// middle of the stream.
typedef __attribute__((ext_vector_type(4))) unsigned int words4;
template <typename P, bool PAST> __device__ __forceinline__ P load_vec(const void *p)
{
    if constexpr (sizeof(P) == 16 && PAST) return __builtin_bit_cast(P, __builtin_nontemporal_load(reinterpret_cast<const words4 *>(p)));
    else if constexpr (sizeof(P) == 4 && PAST) return __builtin_bit_cast(P, __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(p)));
    else return *reinterpret_cast<const P *>(p);
}
template <typename P, bool PAST> __device__ __forceinline__ void store_vec(void *p, const P &v)
{
    if constexpr (sizeof(P) == 16 && PAST) __builtin_nontemporal_store(__builtin_bit_cast(words4, v), reinterpret_cast<words4 *>(p));
    else if constexpr (sizeof(P) == 4 && PAST) __builtin_nontemporal_store(__builtin_bit_cast(unsigned, v), reinterpret_cast<unsigned *>(p));
    else *reinterpret_cast<P *>(p) = v;
}

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }   // nearest even

// exp(d), d in [-128, 88], to the last bits: d log2(e) is rounded at its own size (6e-8 of |d| in the result), so what the product lost goes in behind.
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
__device__ __forceinline__ float exp_full(float d)
{
    constexpr float kLost = 1.92596299e-8f;   // log2(e) - kLog2e
    const float whole = d * kLog2e, x = __builtin_amdgcn_exp2f(whole);
    return fmaf(x, kLn2 * fmaf(d, kLost, fmaf(d, kLog2e, -whole)), x);
}

// A wavefront's sum or maximum by data-parallel moves, a fifth of the time of six exchanges through LDS: within rows of 16 lanes, then
// across rows; lane 63 has the result, which every lane gets.  `none`: what an absent neighbour counts as.
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float v, float none)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <typename F> __device__ __forceinline__ float wave_reduce(float v, float none, F op)
{
    v = op(v, moved<0x111, 0xf>(v, none));   // one, two, four, eight lanes up
    v = op(v, moved<0x112, 0xf>(v, none));
    v = op(v, moved<0x114, 0xf>(v, none));
    v = op(v, moved<0x118, 0xf>(v, none));
    v = op(v, moved<0x142, 0xa>(v, none));   // the last lane of a row to the next row
    v = op(v, moved<0x143, 0xc>(v, none));   // lane 31 to the upper half
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_sum_fast(float v) { return wave_reduce(v, 0.f, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float wave_max_fast(float v) { return wave_reduce(v, -3.402823466e38f, [](float a, float b) { return fmaxf(a, b); }); }

template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double v)
{
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum_fast(double v)
{
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)u, 63), hi = (unsigned)__builtin_amdgcn_readlane((int)(u >> 32), 63);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}

__device__ __forceinline__ unsigned wave_max_fast(unsigned v)
{
    auto up = [&](auto step) { v = max(v, (unsigned)step((int)v)); };
    up([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false); });
    up([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false); });
    up([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false); });
    up([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false); });
    up([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false); });
    up([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false); });
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// Sums over the lanes whose number agrees modulo `period` (a power of two up to 64), in every lane: rotations within rows of 16 lanes, longest
// first, so that each meets the sums that it lacks; then two exchanges across rows.
template <int CTRL, int N> __device__ __forceinline__ void add_moved(float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += moved<CTRL, 0xf>(v[e], 0.f);
}
template <int O, int N> __device__ __forceinline__ void add_exchanged(float (&v)[N])
{
    float w[N];
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = __shfl_xor(v[e], O, 64);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += w[e];
}
template <int N> __device__ __forceinline__ void stride_sums(float (&v)[N], int period)
{
    if (period <= 8) add_moved<0x128>(v);
    if (period <= 4) add_moved<0x124>(v);
    if (period <= 2) add_moved<0x122>(v);
    if (period <= 1) add_moved<0x121>(v);
    if (period <= 16) add_exchanged<16>(v);
    if (period <= 32) add_exchanged<32>(v);
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
