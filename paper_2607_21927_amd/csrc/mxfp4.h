// 4-bit values: E2M1 codes in blocks of 32 that share a power of two (E8M0).
#pragma once

#include "ris_device.h"

namespace ris {
namespace {

constexpr uint32_t kNanScale = 255;

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Scale byte of a block whose largest magnitude has these float32 bits: e + 127
// with e the least with amax <= 7 * 2^e (7 / 4 is mantissa 0x600000), -124..125.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax >= 0x7F800000u) return kNanScale;
    const int e = (int)(amax >> 23) - 2 + ((amax & 0x7FFFFFu) > 0x600000u);
    return (uint32_t)(e < 3 ? 3 : (e > 252 ? 252 : e));
}

// Eight values -> eight codes, the first in the low bits.
__device__ __forceinline__ uint32_t encode8(const float* x, float scale) {
    uint32_t u = 0;
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], scale, 0);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], scale, 1);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], scale, 2);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], scale, 3);
    return u;
}

// Eight codes -> eight bf16 values, exactly.
__device__ __forceinline__ u32x4_t decode8(uint32_t u, float scale) {
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 3))};
}

}  // namespace
}  // namespace ris
