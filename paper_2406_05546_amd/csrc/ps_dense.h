// Shared by the dense-layer and optimizer operators (include/ps_dense.h): element types, loads of any
// alignment, errors.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ps_dense.h"

namespace ps {

struct bf16_t { uint16_t bits; };
struct f16_t { uint16_t bits; };

inline int dtype_size(int dtype) { return dtype == PS_F32 ? 4 : 2; }

ps_status dense_fail(ps_status st, const char* format, ...) __attribute__((format(printf, 2, 3)));

#if defined(__HIPCC__)
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16_t x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_float(f16_t x) { return (float)__builtin_bit_cast(_Float16, x.bits); }

// To the nearest, ties to even; NaN stays NaN.
template <class T>
__device__ __forceinline__ T from_float(float x)
{
    if constexpr (sizeof(T) == 4)
        return x;
    else if constexpr (__is_same(T, bf16_t))
        return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)x)};
    else
        return f16_t{__builtin_bit_cast(uint16_t, (_Float16)x)};
}

// N consecutive elements from or to memory that is aligned to an element only: the hardware takes wide accesses at
// any address, and the compiler makes wide instructions of these copies.
template <int N, class T>
__device__ __forceinline__ void load_n(const T* p, float (&v)[N])
{
    T raw[N];
    __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_float(raw[i]);
}
template <int N, class T>
__device__ __forceinline__ void store_n(T* p, const float (&v)[N])
{
    T raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = from_float<T>(v[i]);
    __builtin_memcpy(p, raw, sizeof(raw));
}
// The first n of them (zeros behind).  The address is hidden from the compiler: next to load_n or store_n of the same elements, in the
// other branch, it would take what both have in common out of both, and leave no wide access in either.
template <int N, class T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[N])
{
    asm volatile("" : "+v"(p));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? to_float(p[i]) : 0.f;
}
template <int N, class T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[N])
{
    asm volatile("" : "+v"(p));
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = from_float<T>(v[i]);
}
#endif

}  // namespace ps
