// What the paged-cache kernels share: 8-bit codes to 16-bit matrix operands,
// argument checks, and the device's size.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <tuple>

#include "../../include/paged_kv.h"

namespace paged {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct E4M3 {};
struct Int8 {};

// The 16-bit matrix type of an activation type: eight elements of one lane.
template <class T>
struct Act;
template <>
struct Act<bf16> {
    typedef bf16x8 frag;
    static __device__ f32x4 mfma16(frag a, frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ f32x16 mfma32(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Act<f16> {
    typedef f16x8 frag;
    static __device__ f32x4 mfma16(frag a, frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ f32x16 mfma32(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

// Four codes of a dword as 16-bit floats, exactly: every e4m3 value and every
// int8 is one of f16 and of bf16.
template <class C, class T>
struct Four;
template <>
struct Four<E4M3, f16> {
    static __device__ u32x2 of(u32 x) {
        return u32x2{__builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.0f, false)),
                     __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.0f, true))};
    }
};
template <>
struct Four<E4M3, bf16> {
    static __device__ u32x2 of(u32 x) {
        return u32x2{__builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.0f, false)),
                     __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.0f, true))};
    }
};
template <>
struct Four<Int8, f16> {
    // code + 128 as the low bits of an f16 in [1024, 2048), less 1152
    static __device__ u32x2 of(u32 x) {
        const u32 u = x ^ 0x80808080u;
        const f16x2 b = {(f16)1152.0f, (f16)1152.0f};
        const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - b;
        const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - b;
        return u32x2{__builtin_bit_cast(u32, lo), __builtin_bit_cast(u32, hi)};
    }
};
template <>
struct Four<Int8, bf16> {
    static __device__ u32x2 of(u32 x) {
        const int s = (int)x;
        const f32x2 a = {(float)(signed char)s, (float)(signed char)(s >> 8)};
        const f32x2 b = {(float)(signed char)(s >> 16), (float)(signed char)(s >> 24)};
        return u32x2{__builtin_bit_cast(u32, __builtin_convertvector(a, bf16x2)),
                     __builtin_bit_cast(u32, __builtin_convertvector(b, bf16x2))};
    }
};

// Eight codes (two dwords) as one lane's operand.
template <class C, class T>
__device__ inline typename Act<T>::frag eight(u32 lo, u32 hi) {
    const u32x2 a = Four<C, T>::of(lo), b = Four<C, T>::of(hi);
    return __builtin_bit_cast(typename Act<T>::frag, u32x4{a[0], a[1], b[0], b[1]});
}

// A 4 x 4 transpose of bytes: out[k] holds byte k of r0, r1, r2, r3.
__device__ inline void transpose4(u32 r0, u32 r1, u32 r2, u32 r3, u32 out[4]) {
    const u32 a = __builtin_amdgcn_perm(r1, r0, 0x05010400u), b = __builtin_amdgcn_perm(r1, r0, 0x07030602u);
    const u32 c = __builtin_amdgcn_perm(r3, r2, 0x05010400u), d = __builtin_amdgcn_perm(r3, r2, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline u32 pack_f16(float a, float b) {
    return __builtin_bit_cast(u32, __builtin_convertvector((f32x2{a, b}), f16x2));
}
template <class T>
__device__ inline u32 pack2(float a, float b);
template <>
__device__ inline u32 pack2<f16>(float a, float b) { return pack_f16(a, b); }
template <>
__device__ inline u32 pack2<bf16>(float a, float b) {
    return __builtin_bit_cast(u32, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// Host side.

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

inline int log2_page(int page) {
    for (int b = 4; b <= 8; ++b)
        if (page == 1 << b) return b;
    return -1;
}

// PAGED_KV_OK where the kernels can read this cache.
inline int check_cache(const paged_kv_cache *c, bool values) {
    if (!c || !c->k || !c->k_scale || !aligned16(c->k)) return PAGED_KV_EINVAL;
    if (values && (!c->v || !c->v_scale || !aligned16(c->v))) return PAGED_KV_EINVAL;
    if (c->n_pages < 1 || c->n_heads < 1) return PAGED_KV_EINVAL;
    if (c->code != PAGED_KV_E4M3 && c->code != PAGED_KV_INT8) return PAGED_KV_EINVAL;
    if (log2_page(c->page) < 0) return PAGED_KV_EUNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return PAGED_KV_EUNSUPPORTED;
    if (c->page_stride < (int64_t)c->n_heads * c->page * c->head_dim || c->page_stride % c->head_dim != 0 ||
        c->scale_stride < c->n_heads)
        return PAGED_KV_EINVAL;
    if ((double)c->n_pages * (double)(c->page_stride / c->head_dim) >= 4294967296.0) return PAGED_KV_EUNSUPPORTED;
    return PAGED_KV_OK;
}

// Compute units of the current device; 0 where it is no gfx950.
inline int device_cus() {
    static int known[64];  // + 1; each written with one value
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
    if (known[dev] == 0) {
        hipDeviceProp_t p;
        if (hipGetDeviceProperties(&p, dev) != hipSuccess) return 0;
        bool gfx950 = true;
        const char *want = "gfx950";
        for (int i = 0; i < 6; ++i) gfx950 = gfx950 && p.gcnArchName[i] == want[i];
        known[dev] = 1 + (gfx950 ? p.multiProcessorCount : 0);
    }
    return known[dev] - 1;
}

// A launch that reports its own status and leaves the thread's last error alone.
template <class... P, class... A>
inline int launch(void (*kernel)(P...), dim3 grid, dim3 block, void *stream, const A &...args) {
    std::tuple<P...> held(args...);
    return std::apply(
        [&](P &...a) {
            void *p[] = {(void *)&a...};
            return hipLaunchKernel((const void *)kernel, grid, block, p, 0, (hipStream_t)stream) == hipSuccess
                       ? PAGED_KV_OK
                       : PAGED_KV_ELAUNCH;
        },
        held);
}

}  // namespace paged
