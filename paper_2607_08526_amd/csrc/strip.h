// The store of a wavefront's strip of accumulators, 32 MS rows by 64 columns in
// 32 x 32 MFMA tiles, through a patch of LDS that only this wavefront uses: a
// store instruction then covers whole 256-byte (fp32) or 128-byte (bf16) pieces
// of four rows.
//
// Loads and stores retire in order: a load behind a store waits until memory has
// taken the store.  So what the epilogue reads of the next row block is loaded before
// a row block's first store, and a strip without an epilogue loads nothing.  (With a load,
// even one that its branch skips, between the stores: 10 us per launch.)
#pragma once

#include "epilogue.h"
#include "gated.h"

namespace qlk {

typedef float strip_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t strip_u32x2 __attribute__((ext_vector_type(2)));
constexpr int STRIP_PATCH = 32 * 64;  // floats of a wavefront's patch

// a plain store but for its type: nothing is loaded
__host__ __device__ inline bool strip_plain(const Epilogue &e)
{
    return !e.bias && !e.resid && !e.steer && !e.act && !e.ycopy;
}

// row block's 32 x 64 accumulators (two MFMA tiles side by side) to the patch
template <typename ACC>
__device__ inline void strip_put(float *patch, int lane, const ACC &left, const ACC &right)
{
    const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        float *const p = patch + (8 * (r >> 2) + 4 * g + (r & 3)) * 64 + l32;
        p[0] = left[r];
        p[32] = right[r];
    }
}

// Y[m0 ..][n0 .. n0 + 63] of an output with an epilogue (EPI) or a plain one; vec:
// groups of four columns (epi_vec_ok); nt: not read again soon.
template <bool EPI, int MS, typename ACC>
__device__ inline void strip_store(const Epilogue &e, float *Y, int M, int N, int m0, int n0,
                                   float *patch, int lane, const ACC (&acc)[MS][2], bool vec,
                                   bool nt)
{
    const int rl = lane >> 4, cq = 4 * (lane & 15), n = n0 + cq;
    strip_f32x4 b4 = {0.f, 0.f, 0.f, 0.f}, s4 = b4;
    float alpha = 0.0f;
    if (EPI && vec && n < N) {
        if (e.bias)
            b4 = *reinterpret_cast<const strip_f32x4 *>(e.bias + n);
        s4 = epi_steer4<strip_f32x4>(e, n, alpha);
    }
    auto put = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        strip_put(patch, lane, acc[i][0], acc[i][1]);
    };
    auto read = [&](int u) {
        return *reinterpret_cast<const strip_f32x4 *>(patch + (4 * u + rl) * 64 + cq);
    };
    // this lane's row of store u of a row block that starts at mb: mb + 4 u
    strip_f32x4 r[8];
    auto load_resid = [&](int mb) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (e.resid && mb + 4 * u < M && n < N)
                r[u] = __builtin_nontemporal_load(reinterpret_cast<const strip_f32x4 *>(
                    e.resid + (int64_t)(mb + 4 * u) * N + n));
    };
    if (EPI && vec) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            r[u] = b4;
        load_resid(m0 + rl);
    }
#pragma unroll 1
    for (int i = 0; i < MS; ++i) {
        static_assert(MS == 2 || MS == 4, "row blocks");
        const int mb = m0 + 32 * i + rl;
        if (i == 0)
            put(std::integral_constant<int, 0>{});
        else if (MS == 2 || i == 1)
            put(std::integral_constant<int, 1>{});
        else if (i == 2)
            put(std::integral_constant<int, MS - 2>{});
        else
            put(std::integral_constant<int, MS - 1>{});
        if (!vec) {
#pragma unroll 1
            for (int u = 0; u < 8; ++u) {
                const int m = mb + 4 * u;
                const strip_f32x4 v = read(u);
                const int64_t at = (int64_t)m * N + n;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (m < M && n + q < N) {
                        if constexpr (EPI)
                            epi_store(e, Y, at + q, n + q, v[q]);
                        else if (e.ybf16)
                            reinterpret_cast<uint16_t *>(Y)[at + q] = (uint16_t)epi_bf16(v[q]);
                        else
                            Y[at + q] = v[q];
                    }
            }
            continue;
        }
        strip_f32x4 w[8];
        epi_u32x2 cp[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            w[u] = read(u);
            if constexpr (EPI) {
                w[u] = epi_apply4(e, w[u], b4, r[u], s4, alpha);
                if (e.ycopy)
                    cp[u] = epi_bf16x4(w[u]);
            }
        }
        if (EPI && i + 1 < MS)
            load_resid(mb + 32);
        if (e.ybf16) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const strip_u32x2 b = {mx_pack_bf16(w[u][0], w[u][1]),
                                       mx_pack_bf16(w[u][2], w[u][3])};
                if (mb + 4 * u < M && n < N)
                    __builtin_nontemporal_store(
                        b, reinterpret_cast<strip_u32x2 *>(reinterpret_cast<uint16_t *>(Y) +
                                                           (int64_t)(mb + 4 * u) * N + n));
            }
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (mb + 4 * u < M && n < N) {
                    const int64_t at = (int64_t)(mb + 4 * u) * N + n;
                    if (nt)
                        __builtin_nontemporal_store(w[u],
                                                    reinterpret_cast<strip_f32x4 *>(Y + at));
                    else
                        *reinterpret_cast<strip_f32x4 *>(Y + at) = w[u];
                    if (EPI && e.ycopy)
                        epi_copy4(e, at, cp[u], true);
                }
        }
    }
}

// The same for a gated pair: acc[i][0] the gate's and acc[i][1] the up
// projection's 32 columns n0 ..  (forward, or with dG the gradients).
template <int MS, typename ACC>
__device__ inline void strip_gated(const GateArgs &t, int M, int N, int m0, int n0, float *patch,
                                   int lane, const ACC (&acc)[MS][2])
{
    const int rl = lane >> 3, n = n0 + 4 * (lane & 7);
    float bg[4], bu[4];
    gate_bias4(t, n, N, bg, bu);
    auto put = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        strip_put(patch, lane, acc[i][0], acc[i][1]);
    };
    float dh[4][4];
    auto load_dh = [&](int mb) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (mb + 8 * u < M && n < N)
                gate_load_dh(t, (int64_t)(mb + 8 * u) * N, n, N, dh[u]);
    };
    if (t.dG)
        load_dh(m0 + rl);
#pragma unroll 1
    for (int i = 0; i < MS; ++i) {
        static_assert(MS == 2 || MS == 4, "row blocks");
        const int mb = m0 + 32 * i + rl;
        if (i == 0)
            put(std::integral_constant<int, 0>{});
        else if (MS == 2 || i == 1)
            put(std::integral_constant<int, 1>{});
        else if (i == 2)
            put(std::integral_constant<int, MS - 2>{});
        else
            put(std::integral_constant<int, MS - 1>{});
        auto pair = [&](int u, float(&g)[4], float(&v)[4]) {
            const float *const p = patch + (8 * u + rl) * 64 + 4 * (lane & 7);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                g[q] = p[q] + bg[q];
                v[q] = p[32 + q] + bu[q];
            }
        };
        if (t.dG) {
            float dc[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    dc[u][q] = dh[u][q];
            if (i + 1 < MS)
                load_dh(mb + 32);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float g[4], v[4];
                pair(u, g, v);
                if (mb + 8 * u < M && n < N)
                    gate_backward(t, (int64_t)(mb + 8 * u) * N, n, N, g, v, dc[u]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float g[4], v[4];
                pair(u, g, v);
                if (mb + 8 * u < M && n < N)
                    gate_forward(t, (int64_t)(mb + 8 * u) * N, n, N, g, v);
            }
        }
    }
}

}  // namespace qlk
