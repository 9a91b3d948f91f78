// 4-bit K/V rows (SG_FP4).
//
// A row of d channels is d / 2 code bytes (channel 2i in the low nibble of
// byte i) and one scale byte per 32 channels.  A code is a sign bit over a
// magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1); a scale byte s stands for
// 2^(s - 127), 255 for NaN (E8M0).  Writing a block with largest magnitude
// `top` takes the smallest 2^e with top <= 7 * 2^e, so the largest value rounds
// to 6 by at most half a step (7 lies half-way to the next magnitude, 8):
// relative error of N(0, 1) rows 0.112 rms, against 0.115 when nothing may
// exceed 6 and 0.115 with e = floor(log2 top) - 2.  The scale is a power of
// two, so x / 2^e is exact and the one rounding is to the nearest code, halves
// to the even one; every stored value is exact in bf16.
#pragma once

#include "sg_internal.h"

namespace sg {

constexpr int FP4_BLOCK = 32;
constexpr uint32_t FP4_NAN_SCALE = 255u;

// Scale byte of a block whose largest magnitude has the float bits `top`
// (sign clear).  Clamped so that every code times the scale is a normal float:
// from 2^-125 (values below round to zero or to steps of 2^-126) to 2^125
// (magnitudes above 6 * 2^125 are stored as that).
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return FP4_NAN_SCALE;      // an infinity or NaN: the block reads as NaN
    const int b = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)min(max(b, 2), 252);
}

__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of 8 consecutive channels, rounded and saturated by the conversion
// instruction (which divides by the scale).
__device__ __forceinline__ uint32_t fp4_encode8(const float (&x)[8], float scale) {
    uint32_t w = 0u;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Channels 2 SEL and 2 SEL + 1 of a word of 8 codes as two bf16 (exact; a
// scale of byte 255 gives NaN).
template <int SEL>
__device__ __forceinline__ uint32_t fp4_bf16_pair(uint32_t codes, float scale) {
    const auto r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL);
    uint32_t w;
    __builtin_memcpy(&w, &r, sizeof(w));
    return w;
}

}  // namespace sg
