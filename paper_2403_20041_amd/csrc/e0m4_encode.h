// Fit and encode steps of the E0M4 quantiser (paper: section "E0M4 FP4 quantization", quantization paragraph), for the files that
// are compiled with -ffp-contract=off: every fp32 step is one IEEE operation (divide, add, compare, convert), which is what makes
// the codes reproducible bit for bit on another machine.
#pragma once

#include "e0m4_device.h"

namespace e0m4 {

constexpr float kLo = 2.0f;             // 2^n with n = 1
constexpr float kHi = 3.998046875f;     // 2^(n+1) - eps, eps = one fp16 ulp of the binade (bits 0x43FF)
constexpr float kSpan = 1.998046875f;   // kHi - kLo, exact
constexpr float kMinScale = 6.103515625e-05f;   // smallest normal fp16
constexpr float kMaxScale = 65504.0f;           // largest finite fp16

__device__ inline uint16_t half_bits(half_t h) { return __builtin_bit_cast(uint16_t, h); }
__device__ inline half_t bits_half(uint16_t b) { return __builtin_bit_cast(half_t, b); }

// code = min(y1 + y2, 15): y1 = four highest fraction bits of the mapped fp16
// value, y2 = the bit below them (paper: quantization paragraph).
// (y1 + y2 is the five bits above bit 5, plus one, halved; every value here lies in [2, 4))
__device__ inline uint32_t encode_value(float w0, const Divisor& sf, float bf)
{
    float q = quotient(w0, sf);
    float t = q + bf;
    t = t < kLo ? kLo : t;
    t = t > kHi ? kHi : t;
    const uint32_t bits = half_bits((half_t)t);
    const uint32_t c = (((bits >> 5) & 31u) + 1u) >> 1;
    return c > 15u ? 15u : c;
}

}  // namespace e0m4
