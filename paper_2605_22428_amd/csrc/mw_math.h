// What the arithmetic operators (gate, experts, adapters) share: types of the matrix instructions, conversions, checks.
#ifndef MW_MATH_H_
#define MW_MATH_H_

#include "mw_internal.h"

// An entry point of a context is called with the context's device current (as everywhere in the library).
static inline int32_t mw_on_device_of(const mw_ctx *ctx)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return MW_ERR_HIP;
    return dev == ctx->device ? MW_OK : MW_ERR_INVALID_ARG;
}

#ifdef __HIPCC__
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float mw_bf16_to_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t mw_f32_to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

template <int kCtrl, int kRows>
__device__ __forceinline__ float mw_dpp_f32(float v)       // lanes without a source get 0
{
    return __uint_as_float(mw_dpp<kCtrl, kRows>(__float_as_uint(v)));
}
// Sum over the wave in a fixed order; every lane active.
__device__ __forceinline__ float mw_wave_sum_f32(float v)
{
    v += mw_dpp_f32<0x111, 0xf>(v);
    v += mw_dpp_f32<0x112, 0xf>(v);
    v += mw_dpp_f32<0x114, 0xf>(v);
    v += mw_dpp_f32<0x118, 0xf>(v);
    v += mw_dpp_f32<0x142, 0xa>(v);
    v += mw_dpp_f32<0x143, 0xc>(v);
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// 32-bit keys that order like the floats they come from, from 1 up; 0 is below every one of them.
__device__ __forceinline__ uint32_t mw_order_key(float v)
{
    const uint32_t b = __float_as_uint(v);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float mw_key_value(uint32_t k) { return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k); }
#endif

#endif  // MW_MATH_H_
