// Activation of a gated feed-forward and its derivative, and the store of the
// outputs that its kernels share.
#pragma once

#include "epilogue.h"
#include "mx.h"

namespace qlk {

// act(g) and act'(g):
//   identity
//   GELU  g Phi(g), Phi + g phi   (Phi as in epi_gelu, phi the normal density)
//   SiLU  g s, s (1 + g (1 - s)),   s = 1 / (1 + exp(-g))
__device__ inline void gate_act(int act, float g, float &a, float &da)
{
    if (act == QL_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
        a = g * s;
        da = s * __builtin_fmaf(g, 1.0f - s, 1.0f);
    } else if (act == QL_ACT_GELU) {
        const float e = __expf(-0.5f * g * g);
        const float z = __builtin_fabsf(g) * 0.70710678118654752f;
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, z, 1.0f));
        float q = __builtin_fmaf(t, 1.061405429f, -1.453152027f);
        q = __builtin_fmaf(t, q, 1.421413741f);
        q = __builtin_fmaf(t, q, -0.284496736f);
        q = __builtin_fmaf(t, q, 0.254829592f);
        q = 0.5f * q * t * e;  // Phi(-|g|)
        const float phi = g >= 0.0f ? 1.0f - q : q;
        a = g * phi;
        da = __builtin_fmaf(g * 0.3989422804014327f, e, phi);
    } else {
        a = g;
        da = 1.0f;
    }
}

// columns n .. n + 3 of a row starting at element `row` of an fp32 or bf16
// output with N columns; vec: whole groups of four at 16- / 8-byte alignment
__device__ inline void gate_store4(void *Y, bool bf16, int64_t row, int n, int N, const float (&v)[4],
                                   bool vec)
{
    if (bf16) {
        uint16_t *const o = static_cast<uint16_t *>(Y) + row + n;
        const uint32_t lo = mx_pack_bf16(v[0], v[1]), hi = mx_pack_bf16(v[2], v[3]);
        if (vec) {
            *reinterpret_cast<uint2 *>(o) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N)
                    o[e] = (uint16_t)((e < 2 ? lo : hi) >> (16 * (e & 1)));
        }
    } else {
        float *const o = static_cast<float *>(Y) + row + n;
        if (vec) {
            *reinterpret_cast<float4 *>(o) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N)
                    o[e] = v[e];
        }
    }
}

// both biases of columns n .. n + 3 (columns past N repeat the last one)
__device__ inline void gate_bias4(const GateArgs &t, int n, int N, float (&bg)[4], float (&bu)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = min(n + e, N - 1);
        bg[e] = t.bias[0] ? t.bias[0][c] : 0.0f;
        bu[e] = t.bias[1] ? t.bias[1][c] : 0.0f;
    }
}

// H = act(g) u of columns n .. n + 3 of the row that starts at element `row`; g,
// u: the two projections with their biases
__device__ inline void gate_forward(const GateArgs &t, int64_t row, int n, int N,
                                    const float (&g)[4], const float (&u)[4])
{
    float h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, da;
        gate_act(t.act, g[e], a, da);
        h[e] = a * u[e];
    }
    gate_store4(t.H, t.hbf16, row, n, N, h, t.vec && n + 3 < N);
}

__device__ inline void gate_load_dh(const GateArgs &t, int64_t row, int n, int N, float (&dh)[4])
{
    const bool vec = t.vec && n + 3 < N;
    if (t.dhbf16) {
        const uint16_t *const p = static_cast<const uint16_t *>(t.dH) + row + n;
        if (vec) {
            const uint2 w = *reinterpret_cast<const uint2 *>(p);
            dh[0] = __uint_as_float(w.x << 16);
            dh[1] = __uint_as_float(w.x & 0xFFFF0000u);
            dh[2] = __uint_as_float(w.y << 16);
            dh[3] = __uint_as_float(w.y & 0xFFFF0000u);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                dh[e] = n + e < N ? __uint_as_float((uint32_t)p[e] << 16) : 0.0f;
        }
    } else {
        const float *const p = static_cast<const float *>(t.dH) + row + n;
        if (vec) {
            const float4 v = *reinterpret_cast<const float4 *>(p);
            dh[0] = v.x;
            dh[1] = v.y;
            dh[2] = v.z;
            dh[3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                dh[e] = n + e < N ? p[e] : 0.0f;
        }
    }
}

// dU = dH act(g), dG = dH u act'(g), rounded once to bf16 (off by at most 2^-8 of each):
// they are operands of bf16 products and outputs, and 16 bits of each are written and
// read back for them.  A gradient of X or of weights then carries independent roundings
// of its terms: 0.0024 of its norm in all with a bf16 output, whose own rounding is
// 0.0017.  (As two bf16 each they would double the matrix instructions.)
__device__ inline void gate_backward(const GateArgs &t, int64_t row, int n, int N,
                                     const float (&g)[4], const float (&u)[4],
                                     const float (&dh)[4])
{
    const bool vec = t.vec && n + 3 < N;
    float dg[4], du[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, da;
        gate_act(t.act, g[e], a, da);
        du[e] = dh[e] * a;
        dg[e] = dh[e] * u[e] * da;
    }
    gate_store4(t.dG, true, row, n, N, dg, vec);
    gate_store4(t.dU, true, row, n, N, du, vec);
}

}  // namespace qlk
