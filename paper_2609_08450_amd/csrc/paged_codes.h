// The scale that 8-bit entries get from their largest magnitude.
#pragma once

#include "paged_common.h"

namespace paged {

constexpr float kLeast = 7.888609052210118e-31f;  // 2^-100

template <class C>
__device__ float scale_of(float top);
template <>
__device__ inline float scale_of<E4M3>(float top) {
    // least power of two s with 448 s >= top; 448 = 1.75 * 2^8
    const u32 b = __float_as_uint(top);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((u32)(max(e, -100) + 127) << 23);
}
template <>
__device__ inline float scale_of<Int8>(float top) { return fmaxf(__fmul_rn(top, 1.0f / 127.0f), kLeast); }

template <class C>
__device__ float value_of(u32 code);
template <>
__device__ inline float value_of<E4M3>(u32 code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }
template <>
__device__ inline float value_of<Int8>(u32 code) { return (float)(signed char)code; }

}  // namespace paged
