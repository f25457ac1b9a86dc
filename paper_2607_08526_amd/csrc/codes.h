// Scales and codes of the int8 and q4 formats, exact without a division: what the
// quantizers (quantize.hip) and the normalisation's int8 outputs (norm.hip) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qlk {

// Exact value of an fp16 bit pattern with the sign bit clear; 0x7C00 as 2^16,
// where the next normal would be.
__device__ inline float f16_value(uint32_t h)
{
    return h >= 0x7C00u ? 65536.0f : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

// fp16 bit pattern nearest to amax / Q for a finite fp32 amax >= 0 (ties to
// even, subnormals kept, 0x7C00 when it rounds past 65504), exact: the fp32
// product with 1 / Q rounds to the right pattern or to a neighbour, and the
// midpoints to both neighbours times Q (12 and 7 significant bits) are exact
// in fp32, to be compared with amax itself.
template <int Q>
__device__ inline uint32_t scale_bits(float amax)
{
    const uint32_t h =
        __builtin_bit_cast(uint16_t, (_Float16)(amax * (1.0f / (float)Q)));  // overflow: 0x7C00
    const float v = f16_value(h);
    const float hi = (v + f16_value(h + 1)) * (0.5f * Q);
    const float lo = (v + f16_value(h - 1)) * (0.5f * Q);
    const bool odd = h & 1;
    if (h < 0x7C00u && (amax > hi || (amax == hi && odd)))
        return h + 1;
    if (h > 0 && (amax < lo || (amax == lo && odd)))
        return h - 1;
    return h;
}

// The integer nearest to w / s, ties to even, clamped to [-Q, Q], for s > 0 an
// fp16 value, |w| < 2^8 s and inv within 2 ulp of 1 / s; exact.  (|w| is at
// most Q (1 + 2^-11) s for a normal scale, and 1.5 Q s for a subnormal one,
// which may round down by a third; the clamp takes the excess.)
//   n = rint(w * inv) is within one of it: the product is off by less than
// 2^-21 of itself, 2^-13.  The remainder r = w - n s, at most s / 2 + 2^-13 s in
// size wherever it decides, is then compared with s / 2: above, n moves towards
// w; at the tie, n moves if it is odd.  r is exact in fp32.  With 2^E <= s <
// 2^(E+1): for n = 0 it is w; otherwise |w| > s / 2 (1 - 2^-21), so w and n s
// are multiples of 2^(E-24) and r, below 2^E, has 24 bits, unless s = 2^E and
// |w| is just below s / 2: there n = +-1 and r rounds to s / 2 or more, and n
// moves to 0 either way, as it has to.
__device__ inline int nearest_code(float w, float s, float inv, float half_s, int Q)
{
    const float n = __builtin_rintf(w * inv);
    const float r = __builtin_fmaf(-n, s, w);
    const float a = __builtin_fabsf(r);
    int c = (int)n;
    if (a > half_s || (a == half_s && (c & 1)))
        c += r > 0.0f ? 1 : -1;
    c = c > Q ? Q : c;
    return c < -Q ? -Q : c;
}

// The same for a bf16 x and Q = 127.  x has 8 significant bits and s 11, so that
// a quotient above 1/4 that is no half-integer is at least 2^-12 from every one
// (170 / 1.9208984375 = 88.50025...), while an fp32 quotient below 2^8 within an
// ulp is within 2^-16 of it; exact half-integers are representable.  One Newton
// step on x * inv with its exact remainder gives the quotient at every
// half-integer, and within an ulp elsewhere.
__device__ inline int nearest_code_bf16(float x, float s, float inv)
{
    const float q = x * inv;
    const float r = __builtin_fmaf(__builtin_fmaf(-q, s, x), inv, q);
    return (int)__builtin_amdgcn_fmed3f(__builtin_rintf(r), -127.0f, 127.0f);
}

// 1 / s for an fp16 s > 0 (2^-24 to 65504, so neither overflows nor underflows)
__device__ inline float inverse(float s) { return __builtin_amdgcn_rcpf(s); }

}  // namespace qlk
