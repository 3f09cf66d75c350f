// Values in 8 bits under a power of two that blocks of 128 of them share: a block's scale, its codes, what they stand for.
#pragma once
#include "../../include/pilc.h"
#include "pilc_fit_device.hpp"

namespace pilc {

constexpr uint32_t kBlock8 = 128;

struct Block8 {
    uint8_t *code, *scale;
    uint64_t stride, scale_stride;
    uint32_t type, shared_bits;  // 2^shared_bits rows share scales
};

// The largest of values by their size, as bits without the sign: NaN is above infinity, and both above all others.
__device__ __forceinline__ uint32_t size_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The byte of the smallest scale under which the largest value is 1.75 times a power of two, 2^8 for E4M3 and 2^15 for E5M2,
// at most: the largest's exponent, one more where its digits are over 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest, uint32_t type)
{
    const int e = (int)((largest + 0x1FFFFFu) >> 23) - (type == PILC_E4M3 ? 8 : 15);
    return largest >= 0x7F800000u ? 255u : (uint32_t)max(e, 0);
}
// What values are multiplied with before they are rounded: 2^(127 - e).
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 254u)) << 23); }
// Four values, already multiplied, as codes; the first in the lowest byte.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, uint32_t type, uint32_t byte)
{
    int v = 0;
    if (type == PILC_E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
    }
    return byte == 255 ? 0x7F7F7F7Fu : (uint32_t)v;
}
// What the codes in a word stand for.
__device__ __forceinline__ void values_of(uint32_t codes, uint32_t type, uint32_t byte, float (&v)[4])
{
    const auto lo = type == PILC_E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false) : __builtin_amdgcn_cvt_pk_f32_bf8((int)codes, false);
    const auto hi = type == PILC_E4M3 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true) : __builtin_amdgcn_cvt_pk_f32_bf8((int)codes, true);
    v[0] = lo[0], v[1] = lo[1], v[2] = hi[0], v[3] = hi[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = byte == 255 ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(v[k], (int)byte - 127);
}

}  // namespace pilc
