// Activations kept in 8 bits (include/ps_dense.h): e4m3 codes, 32 columns of a row sharing a power of two as their scale.
//
// Powers of two cost no precision, only up to one binade of range, and what a code stands for is a value of every type here
// (bf16 always, fp16 in its range) without another rounding.  A lane holds eight consecutive columns, so a block is four lanes.
#pragma once
#include "ps_dense.h"

namespace ps {

constexpr int CHECKPOINT_LANES = PS_CHECKPOINT_BLOCK / 8;

#if defined(__HIPCC__)

// The largest over the four lanes of a quad, all of which take part.
__device__ __forceinline__ uint32_t largest_of_quad(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));  // lanes 1, 0, 3, 2
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));  // lanes 2, 3, 0, 1
}

// The exponent of the largest (by its bits) less 8, one more where it is above 1.75 times its power of two: at most 448 = 1.75 * 2^8 remains.
__device__ __forceinline__ int checkpoint_scale(uint32_t top) { return max((int)((top + 0x1fffffu) >> 23) - 8, 1); }
__device__ __forceinline__ float inverse_of_scale(int scale) { return __uint_as_float((uint32_t)(254 - scale) << 23); }

// A block's largest magnitudes that would be rounded beyond T's largest number (from 248 * 2^8 on to 2^16 in fp16, from 248 * 2^120 on to 2^128
// in the others) are held as 240 times the scale, which is within half a step, too.
template <class T>
constexpr uint32_t CHECKPOINT_LARGE = __is_same(T, f16_t) ? 0x47780000u : 0x7f780000u;  // the bits of those

// The codes of a lane's eight values of type T and the block's scale (2^(scale - 127)).  Columns that are not there are 0.
//
// Most values need a product and a conversion.  Others, those that are not finite, or 0, or so small that their code would be 0, or as large as
// above, are looked for in the largest and smallest magnitudes, and a wavefront that has one takes the way that looks at each value: in the
// layers' kernels, whose last steps are bound by their instructions (8192 rows 2048 -> 8192 with GELU 285 us, 310 where every value is looked at).
template <class T>
__device__ __forceinline__ uint32_t checkpoint_encode(const float (&v)[8], uint32_t (&code)[2])
{
    uint32_t top = 0, low = ~0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
        top = max(top, a);
        low = min(low, a);
    }
    top = largest_of_quad(top);
    int scale = checkpoint_scale(top);
    float inverse = inverse_of_scale(scale), x[8];
    if (__ballot(top >= CHECKPOINT_LARGE<T> || __uint_as_float(low) * inverse < 0x1p-9f)) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
            top = max(top, a < 0x7f800000u ? a : 0u);
        }
        top = largest_of_quad(top);
        scale = checkpoint_scale(top);
        inverse = inverse_of_scale(scale);
        const float most = top >= CHECKPOINT_LARGE<T> ? 240.f : 448.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // what is not 0 is not held as 0: at least 2^-9, the least code; what is not finite as NaN
            const float held = copysignf(fminf(fmaxf(fabsf(v[i] * inverse), 0x1p-9f), most), v[i]);
            x[i] = v[i] == 0.f ? v[i] : (__float_as_uint(v[i]) & 0x7fffffffu) < 0x7f800000u ? held : __uint_as_float(0x7fc00000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[i] * inverse;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int c = 0;
        c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 0], x[4 * i + 1], c, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], c, true);
        code[i] = (uint32_t)c;
    }
    return (uint32_t)scale;
}

__device__ __forceinline__ void checkpoint_decode(const uint32_t (&code)[2], uint32_t scale, float (&v)[8])
{
    const float s = __uint_as_float(scale << 23);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[4 * i + 0] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 0) * s;
        v[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 1) * s;
        v[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 2) * s;
        v[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 3) * s;
    }
}

// `n` codes (8: all) from or to memory of any alignment
__device__ __forceinline__ void load_codes(const uint8_t* p, int n, uint32_t (&code)[2])
{
    if (n >= 8) {
        __builtin_memcpy(code, p, 8);
        return;
    }
    asm volatile("" : "+v"(p));
    code[0] = code[1] = 0;
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) code[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, const uint32_t (&code)[2])
{
    if (n >= 8) {
        __builtin_memcpy(p, code, 8);
        return;
    }
    asm volatile("" : "+v"(p));
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) p[i] = (uint8_t)(code[i / 4] >> (8 * (i % 4)));
}

// Eight columns from `col` (a multiple of 8) of a row, of which `valid` exist: their codes, and once for a block its scale.  Every lane of a
// quad calls this.
template <class T>
__device__ __forceinline__ void checkpoint_store(uint8_t* codes, uint8_t* scales, int col, int valid, const float (&v)[8])
{
    uint32_t code[2];
    const uint32_t scale = checkpoint_encode<T>(v, code);
    if (valid <= 0) return;
    store_codes(codes + col, valid, code);
    if (col % PS_CHECKPOINT_BLOCK == 0) scales[col / PS_CHECKPOINT_BLOCK] = (uint8_t)scale;
}

#endif

}  // namespace ps
