// 4-bit microscaled values (MXFP4): a block of 32 shares a scale 2^(s - 127),
// s one byte (255: NaN), and a code is a sign bit above the magnitudes 0, 0.5,
// 1, 1.5, 2, 3, 4, 6 (one exponent pair, one mantissa bit).  All conversions
// here are single gfx950 instructions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qlinear.h"

namespace qlk {

typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t mx_u32x4 __attribute__((ext_vector_type(4)));

// 2^(s - 127) as an fp32: s = 0 is a subnormal, s = 255 NaN
__device__ inline float mx_scale(uint32_t s)
{
    return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7FC00000u : s << 23);
}

// two fp32 values rounded to nearest even bf16, packed (v_cvt_pk_bf16_f32)
__device__ inline uint32_t mx_pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(mx_f32x2{lo, hi}, mx_bf16x2_t));
}

// the 8 codes of a word times a power of two, as 8 bf16 in k order.  Exact: a
// code has two significant bits and bf16 the exponents of the scale byte
// (magnitudes from 2^128, which only scales that quantization never gives
// reach, are infinite; those below 2^-126 are bf16 subnormals).
__device__ inline mx_u32x4 mx_bf16x8(uint32_t word, float scale)
{
    return mx_u32x4{
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3))};
}

// word w of mx_bf16x8 (w known at compile time)
__device__ inline uint32_t mx_bf16x2(uint32_t word, float scale, int w)
{
    mx_bf16x2_t v;
    switch (w) {
    case 0: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0); break;
    case 1: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1); break;
    case 2: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2); break;
    default: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3); break;
    }
    return __builtin_bit_cast(uint32_t, v);
}

// fp32 weights c * s of 8 q4 codes (one word) or int8 codes (two words): exact for a
// scale as stored (the code has at most 8 significant bits and the scale 11)
__device__ inline void q4_f32x8(uint32_t word, float s, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (float)((int32_t)(word << (28 - 4 * e)) >> 28) * s;
}
__device__ inline void int8_f32x8(uint32_t w0, uint32_t w1, float s, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (float)((int32_t)((e < 4 ? w0 : w1) << (24 - 8 * (e & 3))) >> 24) * s;
}

// A q4 / int8 weight v = c * s as two bf16: hi the leading 8 bits, lo the rest
// rounded to nearest.  Both have v's sign and neither is zero where v is not, so an
// infinite activation meets two infinities of one sign (hi rounded to nearest leaves lo 0
// or of the other sign: NaN).  For that s is taken one fp32 step larger: c times the
// step is more than half a step of c * s, whose 18 bits (q4: 14) end above it, so v
// always has bits behind hi.  Off by at most 2^-16 of c * s for int8, 2^-22 for q4.
__device__ inline float plane_scale(float s) { return __uint_as_float(__float_as_uint(s) | 1u); }
__device__ inline uint32_t plane_hi(float v0, float v1)
{
    return __builtin_amdgcn_perm(__float_as_uint(v1), __float_as_uint(v0), 0x07060302u);
}
__device__ inline uint32_t plane_lo(float v0, float v1)
{
    return mx_pack_bf16(v0 - __uint_as_float(__float_as_uint(v0) & 0xFFFF0000u),
                        v1 - __uint_as_float(__float_as_uint(v1) & 0xFFFF0000u));
}

// word w (two k, w known at compile time) of a run of codes as bf16 planes: raw
// holds 8 codes a word (int8: 4), s is its scale (q4, int8: its plane_scale); MXFP4 has
// one plane, hi
template <int FMT>
__device__ inline void decode_word(const uint32_t *raw, int w, float s, uint32_t &hi, uint32_t &lo)
{
    if constexpr (FMT == QL_FMT_MXFP4) {
        hi = mx_bf16x2(raw[w >> 2], s, w & 3);
        lo = 0;
    } else {
        float v0, v1;
        if constexpr (FMT == QL_FMT_Q4) {
            v0 = (float)((int32_t)(raw[w >> 2] << (28 - 8 * (w & 3))) >> 28);
            v1 = (float)((int32_t)(raw[w >> 2] << (24 - 8 * (w & 3))) >> 28);
        } else {
            v0 = (float)((int32_t)(raw[w >> 1] << (24 - 16 * (w & 1))) >> 24);
            v1 = (float)((int32_t)(raw[w >> 1] << (16 - 16 * (w & 1))) >> 24);
        }
        v0 *= s;
        v1 *= s;
        hi = plane_hi(v0, v1);
        lo = plane_lo(v0, v1);
    }
}

// the planes of 8 weights c * plane_scale(s)
__device__ inline void split2(const float (&v)[8], mx_u32x4 &hi, mx_u32x4 &lo)
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        hi[w] = plane_hi(v[2 * w], v[2 * w + 1]);
        lo[w] = plane_lo(v[2 * w], v[2 * w + 1]);
    }
}

// v as three bf16 planes, packed, largest first: the first two by truncation, so
// that every remainder is exact (|v - sum| <= 2^-27 |v|); an infinity or NaN is
// its own first plane, with nothing behind it
__device__ inline void split3(const float (&v)[8], mx_u32x4 (&p)[3])
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t t[2], u[2];
        float r[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float f = v[2 * w + e];
            const bool fin = __builtin_fabsf(f) < INFINITY;
            t[e] = fin ? __float_as_uint(f) & 0xFFFF0000u : f != f ? 0x7FC00000u : __float_as_uint(f);
            const float q = fin ? f - __uint_as_float(t[e]) : 0.0f;
            u[e] = __float_as_uint(q) & 0xFFFF0000u;
            r[e] = q - __uint_as_float(u[e]);
        }
        p[0][w] = t[0] >> 16 | t[1];
        p[1][w] = u[0] >> 16 | u[1];
        p[2][w] = mx_pack_bf16(r[0], r[1]);
    }
}

}  // namespace qlk
