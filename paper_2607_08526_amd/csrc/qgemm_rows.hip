// Products with MXFP4 weights, and gated pairs of projections in any of the
// quantized formats, without stages in LDS: fp32 activations and gated pairs at few
// rows, where nothing else starts as fast, MXFP4 activations below the tiles of
// qgemm_mx4.hip, and reductions too long for the staged kernels:
//
//   P[m][n] = sum_b sum_{k in b} X[m][k] c[n][k] s[n][b]
//
// Matrix instruction: D[n][m] += W[n][k] X[m][k] by v_mfma_f32_16x16x32_bf16;
// lane l holds row l % 16 of both operands and, of a 128-k step, the whole
// block l / 16 (32 k, in four chunks of 8): its codes are one 16-byte load
// (int8: two), its scale one load, its activations one run of 64 bytes.  The
// sum does not care which k a slot holds as long as both operands agree.
//
// Operand planes keep products as exact as their formats: MXFP4 values are
// exact in bf16; a q4 / int8 weight c * s enters as two bf16 planes (off by at
// most 2^-22 / 2^-16 of itself: mx.h); an fp32 activation as three (exact but for
// what lies below fp32's smallest normal).  MXFP4
// activations meet MXFP4 weights in one v_mfma_scale_f32_16x16x128_f8f6f4 per
// step, which takes codes and scale bytes as they are.
//
// Layout: a workgroup owns 32 weight rows (of a gated pair: the same 16 of
// both) by 16 MT activation rows; its 4 wavefronts take every fourth 128-k
// step, the next one's loads in flight, and add up in LDS at the end.  D^T
// puts 4 consecutive n in a lane: 16-byte stores.
//
// Bound: latency at few rows (a pair of 4096 x 1536 at one row 5.0 us, launch
// included: 6.8 MB are 1.3 us of a copy), the activations re-read per 32 columns
// beyond 64 (MXFP4 6144 x 1536: 16 rows 5.7 us, 64 rows 8.1, 256 rows 13.9 against
// 9.3 on tiles).
#include <algorithm>

#include "epilogue.h"
#include "gated.h"
#include "internal.h"
#include "mx.h"

namespace qlk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;

enum XKind { X_BF16, X_F32, X_MX };

__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int FMT>
struct Wt {
    static constexpr int WORDS = FMT == QL_FMT_INT8 ? 8 : 4;   // of a block's codes
    static constexpr int PLANES = FMT == QL_FMT_MXFP4 ? 1 : 2;
    uint32_t c[WORDS];
    uint32_t s;
};

// the codes and scale of block b of a weight row (beyond the row: zero weights)
template <int FMT>
__device__ inline void load_w(const uint8_t *codes, const void *scales, int64_t row, int nb, int b,
                              Wt<FMT> &w)
{
    const bool in = b < nb;
    const int64_t i = row * nb + (in ? b : 0);
    const u32x4 *const p = reinterpret_cast<const u32x4 *>(codes) + i * (Wt<FMT>::WORDS / 4);
#pragma unroll
    for (int h = 0; h < Wt<FMT>::WORDS / 4; ++h) {
        const u32x4 v = p[h];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w.c[4 * h + e] = in ? v[e] : 0u;
    }
    if constexpr (FMT == QL_FMT_MXFP4)
        w.s = in ? static_cast<const uint8_t *>(scales)[i] : 127u;
    else
        w.s = in ? static_cast<const uint16_t *>(scales)[i] : 0u;
}

// chunk j (8 k) of a block as bf16 planes
template <int FMT>
__device__ inline void weight_planes(const Wt<FMT> &w, int j, float s, u32x4 (&p)[Wt<FMT>::PLANES])
{
    if constexpr (FMT == QL_FMT_MXFP4) {
        p[0] = mx_bf16x8(w.c[j], s);
    } else {
        float v[8];
        if constexpr (FMT == QL_FMT_Q4)
            q4_f32x8(w.c[j], s, v);
        else
            int8_f32x8(w.c[2 * j], w.c[2 * j + 1], s, v);
        split2(v, p[0], p[1]);
    }
}

template <int XK>
struct Xt {
    static constexpr int VECS = XK == X_BF16 ? 4 : XK == X_F32 ? 8 : 1;  // of a block
    u32x4 v[VECS];
    uint32_t s;  // X_MX: scale byte
};

template <int XK>
__device__ inline void load_x(const void *X, const uint8_t *sx, int64_t row, int nb, int b,
                              Xt<XK> &x)
{
    const bool in = b < nb;
    const int64_t i = row * nb + (in ? b : 0);
    const u32x4 *const p = static_cast<const u32x4 *>(X) + i * Xt<XK>::VECS;
#pragma unroll
    for (int h = 0; h < Xt<XK>::VECS; ++h) {
        const u32x4 v = p[h];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x.v[h][e] = in ? v[e] : 0u;
    }
    if constexpr (XK == X_MX)
        x.s = in ? sx[i] : 127u;
}

// chunk j of a block of activations as bf16 planes, largest first
template <int XK, int P>
__device__ inline void act_planes(const Xt<XK> &x, int j, u32x4 (&p)[P])
{
    if constexpr (XK == X_BF16) {
        p[0] = x.v[j];
    } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = __uint_as_float(x.v[2 * j + (e >> 2)][e & 3]);
        split3(v, p);
    }
}

// MT: 16-row activation tiles of a workgroup.  GATED: the two weight tiles are
// the same 16 columns of the gate and of the up projection.
template <int FMT, int XK, bool GATED, int MT>
__global__ __launch_bounds__(THREADS) void qgemm_rows_kernel(const RowsGroup args)
{
    constexpr int XP = XK == X_F32 ? 3 : 1;
    constexpr int SLOTS = 2 * MT * 4;  // accumulators per lane
    __shared__ float red[WAVES][SLOTS][64];
    int li = 0;
#pragma unroll
    for (int i = 1; i < QL_MAX_GROUP; ++i)
        if (i < args.n && (int)blockIdx.x >= args.begin[i])
            li = i;
    const RowsArgs &a = args.d[li];
    // each XCD takes a contiguous range of the layer's tiles, row tiles fastest:
    // the workgroups that read one weight tile share an L2
    const int p = (int)blockIdx.x - args.begin[li], G = args.begin[li + 1] - args.begin[li];
    const int gq = G >> 3, gr = G & 7, xcd = p & 7, idx = p >> 3;
    const int tile = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int M = a.M, N = a.N, nb = a.K >> 5;
    const int tiles_m = (M + 16 * MT - 1) / (16 * MT);
    const int tn = tile / tiles_m, tm = tile - tn * tiles_m;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int n0 = tn * (GATED ? 16 : 32), m0 = tm * 16 * MT;

    const uint8_t *const wc[2] = {a.codes[0], a.codes[GATED ? 1 : 0]};
    const void *const ws[2] = {a.scales[0], a.scales[GATED ? 1 : 0]};
    int64_t wrow[2], xrow[MT];
#pragma unroll
    for (int j = 0; j < 2; ++j)  // rows past N repeat the last one
        wrow[j] = min(n0 + (GATED ? 0 : 16 * j) + l16, N - 1);
#pragma unroll
    for (int i = 0; i < MT; ++i)
        xrow[i] = min(m0 + 16 * i + l16, M - 1);

    f32x4 acc[2][MT];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i)
            acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int steps = (nb + 3) >> 2;
    Wt<FMT> w[2];
    Xt<XK> x[MT];
    auto load = [&](int s) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            load_w<FMT>(wc[j], ws[j], wrow[j], nb, 4 * s + g, w[j]);
#pragma unroll
        for (int i = 0; i < MT; ++i)
            load_x<XK>(a.X, a.sx, xrow[i], nb, 4 * s + g, x[i]);
    };
    if (wave < steps)
        load(wave);
    for (int s = wave; s < steps; s += WAVES) {
        Wt<FMT> wn[2] = {w[0], w[1]};
        Xt<XK> xn[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
            xn[i] = x[i];
        if (s + WAVES < steps)
            load(s + WAVES);
        if constexpr (XK == X_MX) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const i32x8 A = {(int)wn[j].c[0], (int)wn[j].c[1], (int)wn[j].c[2],
                                     (int)wn[j].c[3], 0, 0, 0, 0};
                    const i32x8 B = {(int)xn[i].v[0][0], (int)xn[i].v[0][1], (int)xn[i].v[0][2],
                                     (int)xn[i].v[0][3], 0, 0, 0, 0};
                    acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        A, B, acc[j][i], 4, 4, 0, (int)wn[j].s, 0, (int)xn[i].s);
                }
        } else {
            float sc[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                sc[j] = FMT == QL_FMT_MXFP4
                            ? mx_scale(wn[j].s)
                            : plane_scale((float)__builtin_bit_cast(_Float16, (uint16_t)wn[j].s));
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                u32x4 xp[MT][XP];
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    act_planes<XK, XP>(xn[i], c, xp[i]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    u32x4 wp[Wt<FMT>::PLANES];
                    weight_planes<FMT>(wn[j], c, sc[j], wp);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int q = XP - 1; q >= 0; --q)
#pragma unroll
                            for (int v = Wt<FMT>::PLANES - 1; v >= 0; --v)
                                acc[j][i] = mfma16(wp[v], xp[i][q], acc[j][i]);
                }
            }
        }
    }

    // the wavefronts' sums, in wavefront order: slot (j, i, r) of lane l
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                red[wave][(j * MT + i) * 4 + r][lane] = acc[j][i][r];
    __syncthreads();
    auto total = [&](int j, int i, float (&v)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int slot = (j * MT + i) * 4 + r;
            v[r] = ((red[0][slot][lane] + red[1][slot][lane]) + red[2][slot][lane]) +
                   red[3][slot][lane];
        }
    };
    // register r of lane l: weight row 4 (l / 16) + r, activation row l % 16
    if constexpr (GATED) {
        const int n = n0 + 4 * g;
#pragma unroll
        for (int i = wave; i < MT; i += WAVES) {
            const int m = m0 + 16 * i + l16;
            float gv[4], uv[4];
            total(0, i, gv);
            total(1, i, uv);
            if (m >= M || n >= N)
                continue;
            float bg[4], bu[4], dh[4];
            gate_bias4(a.gate, n, N, bg, bu);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gv[e] += bg[e];
                uv[e] += bu[e];
            }
            const int64_t row = (int64_t)m * N;
            if (a.gate.dG) {
                gate_load_dh(a.gate, row, n, N, dh);
                gate_backward(a.gate, row, n, N, gv, uv, dh);
            } else {
                gate_forward(a.gate, row, n, N, gv, uv);
            }
        }
    } else {
        const bool vec = epi_vec_ok(a.ep, a.Y, N);
#pragma unroll
        for (int t = wave; t < 2 * MT; t += WAVES) {
            const int j = t / MT, i = t - j * MT;
            const int m = m0 + 16 * i + l16, n = n0 + 16 * j + 4 * g;
            float v[4];
            total(j, i, v);
            if (m >= M || n >= N)
                continue;
            const int64_t at = (int64_t)m * N + n;
            if (vec) {
                epi_store4(a.ep, a.Y, at, n, f32x4{v[0], v[1], v[2], v[3]}, false);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < N)
                        epi_store(a.ep, a.Y, at + e, n + e, v[e]);
            }
        }
    }
}

template <int FMT, int XK, bool GATED>
void launch(RowsGroup &g, int maxM, hipStream_t stream)
{
    // (more than 16 rows of other activations: only where the reduction is longer
    // than the staged kernels take)
    const int mt = XK != X_MX || maxM <= 16 ? 1 : maxM <= 32 ? 2 : 4;
    int64_t total = 0;
    for (int i = 0; i < g.n; ++i) {
        g.begin[i] = (int)total;
        total += ((int64_t)g.d[i].M + 16 * mt - 1) / (16 * mt) *
                 (((int64_t)g.d[i].N + (GATED ? 15 : 31)) / (GATED ? 16 : 32));
    }
    for (int i = g.n; i <= QL_MAX_GROUP; ++i)
        g.begin[i] = (int)total;
    const dim3 grid((unsigned)total), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, g); };
    if constexpr (XK == X_MX) {
        if (mt == 2)
            return go(qgemm_rows_kernel<FMT, XK, GATED, 2>);
        if (mt == 4)
            return go(qgemm_rows_kernel<FMT, XK, GATED, 4>);
    }
    go(qgemm_rows_kernel<FMT, XK, GATED, 1>);
}

}  // namespace

int64_t rows_tiles(int64_t M, int64_t N, bool gated)
{
    return (M + 15) / 16 * ((N + (gated ? 15 : 31)) / (gated ? 16 : 32));
}

hipError_t launch_qgemm_rows(int fmt, bool xf32, RowsGroup &g, hipStream_t stream)
{
    const int maxM = g.maxM;
    const bool gated = g.d[0].codes[1] != nullptr;
    if (gated) {
        if (fmt == QL_FMT_MXFP4)
            launch<QL_FMT_MXFP4, X_BF16, true>(g, maxM, stream);
        else if (fmt == QL_FMT_Q4)
            launch<QL_FMT_Q4, X_BF16, true>(g, maxM, stream);
        else
            launch<QL_FMT_INT8, X_BF16, true>(g, maxM, stream);
    } else if (g.d[0].sx) {
        launch<QL_FMT_MXFP4, X_MX, false>(g, maxM, stream);
    } else if (xf32) {
        launch<QL_FMT_MXFP4, X_F32, false>(g, maxM, stream);
    } else {
        launch<QL_FMT_MXFP4, X_BF16, false>(g, maxM, stream);
    }
    return hipGetLastError();
}

}  // namespace qlk
