// Products with MXFP4 weights, and gated pairs of projections in any of the
// quantized formats, for few to a few hundred activation rows: one launch and no
// partial sums in memory.
//
//   P[m][n] = sum_b s[n][b] sum_{k in b} X[m][k] c[n][k]
//
// As in the K-group kernel of the other formats (qgemm_kg.hip), the 16 wavefronts
// of a workgroup cut K among themselves: KG groups of WN wavefronts own the same
// output tile, each its share of every stage's blocks, and add their sums through
// LDS in group order at the end.  What differs: a gated pair's wavefront owns 32
// columns of both projections, whose sums meet in one thread; MXFP4 codes become
// exact bf16 with their scale in one instruction per pair and accumulate in the
// matrix cores, with no work per block (q4 and int8: exact codes, then acc += s *
// partial in fp32); a block's scale travels by itself, so that K % 32 == 0 and scales
// of any alignment are enough.
//
// Memory.  Activations, codes and scales of a stage (256 or 512 k) go to LDS by
// direct-to-LDS loads, at least 128 contiguous bytes per row but for the scales,
// through a ring of NST stages; the loads of a stage go out spread over the step
// before.  Up to 32 rows only the first XR = 8, 16 or 32 are staged: the MFMA's
// other rows repeat them and are never stored.
//
// Contraction.  Per 32-k block and 32 x 32 tile two v_mfma_f32_32x32x16_bf16 over k
// = 32 b + 16 g + 8 h + e (lane group g = lane / 32, chunk h, element e).  fp32
// activations enter as three bf16 planes, as in qgemm_rows.hip.
//
// Bound: latency of a launch, a first stage and the sums (about 5 us) at few rows,
// then the decoding beside the MFMAs.  6144 x 1536: one row 5.4 us, 128 rows 9.0, 256
// rows 12.4; fp32 1000 x 1056 at 77 rows 8.9 us; a q4 pair of 2752 x 1024 at 107 rows
// with both gradients 12.6 us.  A launch holds all shapes of its rows, with the registers
// and LDS of the largest; pairs of more than 32 rows spill (MXFP4 4 registers, int8 22,
// q4 28: the 64-row shapes at 128 registers, 16 wavefronts).
#include <algorithm>
#include <cmath>

#include "dma.h"
#include "gated.h"
#include "internal.h"
#include "mx.h"

namespace qlk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 16, NT = 64 * WAVES;

// NW: weights a wavefront holds 32 rows of (a gated pair: 2).  XR: activation rows
// staged; WN: wavefronts across the columns; BPW: blocks of a stage per wavefront.
template <int FMT_, bool XF32_, int NW_, int XR_, int WN_, int BPW_>
struct Geo {
    static constexpr int FMT = FMT_, NW = NW_, XR = XR_, WN = WN_, BPW = BPW_;
    static constexpr bool XF32 = XF32_, MX = FMT == QL_FMT_MXFP4, I8 = FMT == QL_FMT_INT8;
    static constexpr int MI = XR > 32 ? XR / 32 : 1;  // MFMA row blocks
    static constexpr int KG = WAVES / WN;
    static constexpr int TM = XR, TN = 32 * WN;       // outputs of the tile
    static constexpr int TW = TN * NW;                // weight rows, those of one wavefront
                                                      // together
    static constexpr int EB = KG * BPW;               // 32-k blocks per stage
    static constexpr int XRB = EB * (XF32 ? 128 : 64), XCH = XRB / 16;  // activation bytes,
                                                                        // chunks per row
    static constexpr int CRB = EB * (I8 ? 32 : 16), CCH = CRB / 16;
    static constexpr int SD = EB;                     // scales (a dword each) per weight row
    static constexpr int XBYTES = XR * XRB, CBYTES = TW * CRB, SBYTES = TW * SD * 4;
    // loads in units of one wavefront (1 KB; scales 256 bytes); wavefront w takes
    // units w, w + 16, ..., the last ones repeated so that every wavefront counts the
    // same
    static constexpr int XU = XBYTES / 1024, CU = CBYTES / 1024, SU = (SBYTES + 255) / 256;
    static constexpr int UNITS = XU + CU + SU, LOADS = (UNITS + WAVES - 1) / WAVES;
    static constexpr int RED = KG * TM * TN * 4;      // the groups' sums of one projection
    static constexpr int SLOT = XBYTES + CBYTES + SU * 256;
    static constexpr int NST = std::min(3, 160 * 1024 / SLOT), RING = NST * SLOT;
    static_assert(NST >= 2, "a stage ahead");
    static constexpr int LDS = RING > RED ? RING : RED;
    static_assert(EB % 8 == 0 && XBYTES % 1024 == 0 && CBYTES % 1024 == 0, "whole loads");
    static_assert(LDS <= 160 * 1024, "LDS of a CU");
    static_assert(!XF32 || (MX && NW == 1), "forms built");
};

// chunk swizzles (physical = logical ^ swizzle): the fragment reads of 16 lanes
// (rows, one logical chunk) fall on distinct banks
__device__ inline int xswz(int row) { return row & 15; }
template <int CCH>
__device__ inline int cswz(int row)
{
    return CCH >= 16 ? row & 15 : (row >> 1) & 7;  // 128-byte rows: two per bank row
}

__device__ inline f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 8 codes as bf16 integers in k order (q4: times 16, taken out of the scale)
__device__ inline uint32_t bf16_pair(float lo, float hi)  // of values that bf16 holds exactly
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ inline float sbyte(uint32_t w, int i) { return (float)((int)(w << (24 - 8 * i)) >> 24); }
__device__ inline u32x4 codes_int8(uint32_t w0, uint32_t w1)
{
    return u32x4{bf16_pair(sbyte(w0, 0), sbyte(w0, 1)), bf16_pair(sbyte(w0, 2), sbyte(w0, 3)),
                 bf16_pair(sbyte(w1, 0), sbyte(w1, 1)), bf16_pair(sbyte(w1, 2), sbyte(w1, 3))};
}
__device__ inline u32x4 codes_q4(uint32_t w)
{
    const uint32_t e = (w << 4) & 0xF0F0F0F0u, o = w & 0xF0F0F0F0u;  // even, odd k
    return u32x4{bf16_pair(sbyte(e, 0), sbyte(o, 0)), bf16_pair(sbyte(e, 1), sbyte(o, 1)),
                 bf16_pair(sbyte(e, 2), sbyte(o, 2)), bf16_pair(sbyte(e, 3), sbyte(o, 3))};
}

// One output tile of layer d.
template <class G>
__device__ inline void kgm_tile(const RowsArgs &d, int tile, uint8_t *ring)
{
    constexpr int MI = G::MI, NW = G::NW, XB = G::XF32 ? 4 : 2;
    const int M = d.M, N = d.N, K = d.K, nb = K >> 5;
    const int tiles_m = (M + G::TM - 1) / G::TM;
    const int tn = tile / tiles_m, tm = tile - tn * tiles_m;
    const int m0 = tm * G::TM, n0 = tn * G::TN;
    constexpr int SB = G::MX ? 1 : 2;  // bytes of a scale
    const int crow = nb * (G::I8 ? 32 : 16), srow = nb * SB;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave / G::WN, wn = wave % G::WN;

    // this wavefront's loads: per unit a base, a per-lane offset within the stage's
    // rows, and the bytes a stage advances.  Rows past M and N repeat the last one;
    // chunks past K (a part-filled last stage) the last chunk, and are not used.
    // Weight row r of the tile: output column (r / (32 NW)) * 32 + r % 32 of
    // projection r / 32 % NW.
    auto column = [&](int r) { return n0 + r / (32 * NW) * 32 + (r & 31); };
    const uint8_t *ub[G::LOADS];
    uint32_t urow[G::LOADS];
    int ucol[G::LOADS], ustep[G::LOADS], ulim[G::LOADS];
    uint32_t udst[G::LOADS];
#pragma unroll
    for (int q = 0; q < G::LOADS; ++q) {
        const int u = min(q * WAVES + wave, G::UNITS - 1);  // wave-uniform
        if (u < G::XU) {
            const int slot = u * 64 + lane, row = slot / G::XCH;
            ub[q] = static_cast<const uint8_t *>(d.X) + (int64_t)m0 * K * XB;
            urow[q] = (uint32_t)((min(m0 + row, M - 1) - m0) * K * XB);
            ucol[q] = ((slot % G::XCH) ^ xswz(row)) * 16;
            ustep[q] = G::XRB;
            ulim[q] = K * XB - 16;
            udst[q] = u * 1024;
        } else if (u < G::XU + G::CU) {
            // (a unit's 64 chunks lie in rows of one projection: 8 rows or fewer)
            const int slot = (u - G::XU) * 64 + lane, row = slot / G::CCH;
            const int pj = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(row / 32 % NW);
            ub[q] = d.codes[pj] + (int64_t)n0 * crow;
            urow[q] = (uint32_t)((min(column(row), N - 1) - n0) * crow);
            ucol[q] = ((slot % G::CCH) ^ cswz<G::CCH>(row)) * 16;
            ustep[q] = G::CRB;
            ulim[q] = crow - 16;
            udst[q] = u * 1024;
        } else {
            // scales: [block][TW] of a dword each
            const int slot = ((u - G::XU - G::CU) * 64 + lane) % (G::TW * G::SD);
            ub[q] = nullptr;
            urow[q] = 0;
            ucol[q] = slot / G::TW * SB;
            ustep[q] = G::SD * SB;
            ulim[q] = srow - SB;
            udst[q] = G::XBYTES + G::CBYTES + (u - G::XU - G::CU) * 256;
        }
    }
    // the scale rows of this lane's units (row depends on the unit only through TW)
    const uint8_t *sp[G::LOADS];
#pragma unroll
    for (int q = 0; q < G::LOADS; ++q) {
        const int u = min(q * WAVES + wave, G::UNITS - 1);
        const int slot = (max(u - G::XU - G::CU, 0) * 64 + lane) % (G::TW * G::SD);
        const int row = slot % G::TW;
        sp[q] = static_cast<const uint8_t *>(d.scales[NW == 1 ? 0 : row / 32 % NW]) +
                (int64_t)min(column(row), N - 1) * srow;
    }
    const int iters = (nb + G::EB - 1) / G::EB;
    auto issue = [&](int it, int q) {
        const uint32_t to = dma_lds(ring + (it % G::NST) * G::SLOT) + udst[q];
        const uint32_t col = (uint32_t)min(it * ustep[q] + ucol[q], ulim[q]);
        if (min(q * WAVES + wave, G::UNITS - 1) < G::XU + G::CU)
            dma_load16(ub[q], urow[q] + col, to);
        else
            dma_load_small_at<SB>(sp[q] + col, to);
    };
#pragma unroll
    for (int it = 0; it < G::NST - 1; ++it)
        if (it < iters)
#pragma unroll
            for (int q = 0; q < G::LOADS; ++q)
                issue(it, q);

    // accumulator registers that hold staged rows: 8 (r / 4) + 4 g + r % 4
    constexpr int AR = G::XR < 32 ? G::XR / 2 : 16;
    f32x16 acc[NW][MI];
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < MI; ++i)
            acc[w][i] = f32x16{};

    auto step = [&](int it, auto refill) {
        constexpr bool REFILL = decltype(refill)::value;
        // every LDS read of the previous stage has completed; this one landed
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if constexpr (REFILL)
            __builtin_amdgcn_s_waitcnt(dma_vmcnt((G::NST - 2) * G::LOADS));
        else
            dma_wait<G::LOADS, G::NST - 2>(iters - 1 - it);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // no LDS read moves above the barrier
        const uint8_t *const st = ring + (it % G::NST) * G::SLOT;
#pragma unroll
        for (int u = 0; u < G::BPW; ++u) {
            const int b = kg * G::BPW + u;  // block of the stage
            // past K (the last stage only, which refills nothing)
            if constexpr (!REFILL)
                if (it * G::EB + b >= nb)
                    continue;
            if constexpr (REFILL)
#pragma unroll
                for (int q = u; q < G::LOADS; q += G::BPW)
                    issue(it + G::NST - 1, q);
            u32x4 wv[NW][2];
            float s[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const int wr = (wn * NW + w) * 32 + l32;
                const uint8_t *const wrow = st + G::XBYTES + wr * G::CRB;
                const uint8_t *const sd = st + G::XBYTES + G::CBYTES;
                const uint32_t e = *reinterpret_cast<const uint32_t *>(sd + (b * G::TW + wr) * 4);
                if constexpr (G::MX) {
                    const float f = mx_scale(e);
                    const u32x2 c = *reinterpret_cast<const u32x2 *>(
                        wrow + (b ^ cswz<G::CCH>(wr)) * 16 + 8 * g);
                    wv[w][0] = mx_bf16x8(c[0], f);
                    wv[w][1] = mx_bf16x8(c[1], f);
                } else {
                    s[w] = (float)__builtin_bit_cast(_Float16, (uint16_t)e) *
                           (G::I8 ? 1.0f : 0.0625f);  // exact
                    if constexpr (G::I8) {
                        const u32x4 c = *reinterpret_cast<const u32x4 *>(
                            wrow + ((2 * b + g) ^ cswz<G::CCH>(wr)) * 16);
                        wv[w][0] = codes_int8(c[0], c[1]);
                        wv[w][1] = codes_int8(c[2], c[3]);
                    } else {
                        const u32x2 c = *reinterpret_cast<const u32x2 *>(
                            wrow + (b ^ cswz<G::CCH>(wr)) * 16 + 8 * g);
                        wv[w][0] = codes_q4(c[0]);
                        wv[w][1] = codes_q4(c[1]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int xr = 32 * i + (l32 & (G::XR < 32 ? G::XR - 1 : 31));
                const uint8_t *const xrow = st + xr * G::XRB;
                if constexpr (G::XF32) {
                    u32x4 p[2][3];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int lc = 8 * b + 4 * g + 2 * h;
                        float v[8];
                        *reinterpret_cast<f32x4 *>(v) =
                            *reinterpret_cast<const f32x4 *>(xrow + (lc ^ xswz(xr)) * 16);
                        *reinterpret_cast<f32x4 *>(v + 4) =
                            *reinterpret_cast<const f32x4 *>(xrow + ((lc + 1) ^ xswz(xr)) * 16);
                        split3(v, p[h]);
                    }
#pragma unroll
                    for (int q = 2; q >= 0; --q)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            acc[0][i] = mfma(p[h][q], wv[0][h], acc[0][i]);
                } else {
                    u32x4 a[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        a[h] = *reinterpret_cast<const u32x4 *>(
                            xrow + ((4 * b + 2 * g + h) ^ xswz(xr)) * 16);
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        if constexpr (G::MX) {
                            acc[w][i] = mfma(a[0], wv[w][0], acc[w][i]);
                            acc[w][i] = mfma(a[1], wv[w][1], acc[w][i]);
                        } else {
                            f32x16 p = mfma(a[0], wv[w][0], f32x16{});
                            p = mfma(a[1], wv[w][1], p);
#pragma unroll
                            for (int r = 0; r < AR; ++r)
                                acc[w][i][r] = __builtin_fmaf(s[w], p[r], acc[w][i][r]);
                        }
                    }
                }
            }
        }
    };
    int it = 0;
#pragma unroll 1
    for (; it + G::NST - 1 < iters; ++it)
        step(it, std::true_type{});
#pragma unroll 1
    for (; it < iters; ++it)
        step(it, std::false_type{});

    // The groups' sums as rows in LDS, one projection after the other (every stage
    // issued has been waited for and, behind the barrier, read), then every thread
    // adds groups of four columns.
    float *const red = reinterpret_cast<float *>(ring);
    constexpr int ROUNDS = (G::TM * G::TN / 4 + NT - 1) / NT;
    f32x4 v[NW][ROUNDS];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int r = 0; r < AR; ++r)
                red[(kg * G::TM + 32 * i + 8 * (r >> 2) + 4 * g + (r & 3)) * G::TN + wn * 32 + l32] =
                    acc[w][i][r];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < ROUNDS; ++t) {
            const int q = tid + t * NT;
            if (q >= G::TM * G::TN / 4)
                continue;
            const f32x4 *const src = reinterpret_cast<const f32x4 *>(red) + q;
            f32x4 sum = src[0];
#pragma unroll
            for (int k = 1; k < G::KG; ++k)
                sum += src[k * (G::TM * G::TN / 4)];
            v[w][t] = sum;
        }
    }
    const bool vec = NW == 1 && epi_vec_ok(d.ep, d.Y, N);
#pragma unroll
    for (int t = 0; t < ROUNDS; ++t) {
        const int q = tid + t * NT;
        const int m = m0 + q / (G::TN / 4), n = n0 + 4 * (q % (G::TN / 4));
        if (q >= G::TM * G::TN / 4 || m >= M || n >= N)
            continue;
        const int64_t row = (int64_t)m * N;
        if constexpr (NW == 2) {
            float bg[4], bu[4], gv[4], uv[4];
            gate_bias4(d.gate, n, N, bg, bu);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gv[e] = v[0][t][e] + bg[e];
                uv[e] = v[NW - 1][t][e] + bu[e];
            }
            if (d.gate.dG) {
                float dh[4];
                gate_load_dh(d.gate, row, n, N, dh);
                gate_backward(d.gate, row, n, N, gv, uv, dh);
            } else {
                gate_forward(d.gate, row, n, N, gv, uv);
            }
        } else if (vec) {
            epi_store4(d.ep, d.Y, row + n, n, v[0][t], false);
        } else {
#pragma unroll 1
            for (int e = 0; e < 4 && n + e < N; ++e)
                epi_store(d.ep, d.Y, row + n + e, n + e, v[0][t][e]);
        }
    }
}

// The shapes a launch may mix: XR = 8, 16 or 32 for launches of at most that many
// rows (of bf16) and 64 above.  fp32: row tiles of 16 and 32.
template <int FMT, bool XF32, int NW, int XR>
struct Shapes {
    static constexpr int XR1 = XF32 ? 32 : XR < 32 ? XR : 32;
    static constexpr bool R2 = !XF32 && XR > 32;
    // (256 int8 rows of a pair leave no room for a second stage; a pair's 64 x 128
    // of q4 not enough registers)
    static constexpr bool W4 = FMT != QL_FMT_INT8 || NW == 1;
    static constexpr bool RW4 = R2 && W4 && (FMT != QL_FMT_Q4 || NW == 1);
    using R1W4 = Geo<FMT, XF32, NW, XR1, W4 ? 4 : 2, W4 ? 2 : 1>;
    using R1W2 = Geo<FMT, XF32, NW, XR1, 2, 1>;
    using R1W1 = Geo<FMT, XF32, NW, XF32 ? 16 : XR1, 1, 1>;
    using R2W4 = Geo<FMT, XF32, NW, XF32 ? 32 : 64, W4 ? 4 : 2, W4 ? 2 : 1>;
    using R2W2 = Geo<FMT, XF32, NW, XF32 ? 32 : 64, 2, 1>;
};

template <class S>
constexpr int shapes_lds()
{
    int v = std::max(S::R1W4::LDS, std::max(S::R1W2::LDS, S::R1W1::LDS));
    return S::R2 ? std::max(v, std::max(S::R2W4::LDS, S::R2W2::LDS)) : v;
}

template <class S>
__global__ __launch_bounds__(NT, 4) void qgemm_kgm_kernel(const RowsGroup args)
{
    __shared__ __align__(16) uint8_t ring[shapes_lds<S>()];
    int li = 0;
#pragma unroll
    for (int i = 1; i < QL_MAX_GROUP; ++i)
        if (i < args.n && (int)blockIdx.x >= args.begin[i])
            li = i;
    const RowsArgs &d = args.d[li];
    // each XCD takes a contiguous range of the layer's tiles, row tiles fastest
    const int p = (int)blockIdx.x - args.begin[li], G = args.begin[li + 1] - args.begin[li];
    const int gq = G >> 3, gr = G & 7, xcd = p & 7, idx = p >> 3;
    const int tile = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    switch (d.shape) {
    case KGM_R1W1:
        kgm_tile<typename S::R1W1>(d, tile, ring);
        break;
    case KGM_R1W2:
        kgm_tile<typename S::R1W2>(d, tile, ring);
        break;
    case KGM_R1W4:
        if constexpr (S::W4)
            kgm_tile<typename S::R1W4>(d, tile, ring);
        break;
    case KGM_R2W2:
        if constexpr (S::R2)
            kgm_tile<typename S::R2W2>(d, tile, ring);
        break;
    default:
        if constexpr (S::RW4)
            kgm_tile<typename S::R2W4>(d, tile, ring);
    }
}

// rows and columns of a shape's tile ({0, 0}: the launch has no such shape)
template <class S>
KgTile tile_of(int shape)
{
    switch (shape) {
    case KGM_R1W1: return KgTile{S::R1W1::TM, S::R1W1::TN};
    case KGM_R1W2: return KgTile{S::R1W2::TM, S::R1W2::TN};
    case KGM_R1W4: return S::W4 ? KgTile{S::R1W4::TM, S::R1W4::TN} : KgTile{0, 0};
    case KGM_R2W2: return S::R2 ? KgTile{S::R2W2::TM, S::R2W2::TN} : KgTile{0, 0};
    default: return S::RW4 ? KgTile{S::R2W4::TM, S::R2W4::TN} : KgTile{0, 0};
    }
}

// f(Shapes<...>{}) of a launch
template <int FMT, bool XF32, int NW, typename F>
auto with_rows(int maxM, F f)
{
    if constexpr (XF32)
        return f(Shapes<FMT, true, NW, 32>{});
    else
        return maxM > 32   ? f(Shapes<FMT, false, NW, 64>{})
               : maxM > 16 ? f(Shapes<FMT, false, NW, 32>{})
               : maxM > 8  ? f(Shapes<FMT, false, NW, 16>{})
                           : f(Shapes<FMT, false, NW, 8>{});
}
template <typename F>
auto with_shapes(int fmt, bool xf32, bool gated, int maxM, F f)
{
    if (!gated)
        return xf32 ? with_rows<QL_FMT_MXFP4, true, 1>(maxM, f)
                    : with_rows<QL_FMT_MXFP4, false, 1>(maxM, f);
    return fmt == QL_FMT_MXFP4 ? with_rows<QL_FMT_MXFP4, false, 2>(maxM, f)
           : fmt == QL_FMT_Q4  ? with_rows<QL_FMT_Q4, false, 2>(maxM, f)
                               : with_rows<QL_FMT_INT8, false, 2>(maxM, f);
}

}  // namespace

KgTile kgm_tile_shape(int fmt, bool xf32, bool gated, int64_t maxM, int shape)
{
    return with_shapes(fmt, xf32, gated, (int)maxM,
                       [&](auto s) { return tile_of<decltype(s)>(shape); });
}

bool kgm_takes(int64_t K) { return K < ((int64_t)1 << 22); }

// us of a workgroup of each shape: fixed, and per 256 k (measured on layers of K =
// 1024 to 6144, one and many rounds of workgroups).  Products of bf16 and of fp32
// activations with MXFP4 weights, gated pairs of MXFP4, q4 and int8.
struct Rate {
    double fixed, per256;
};
constexpr Rate RATES[5][KGM_SHAPES] = {
    {{2.6, 0.25}, {2.7, 0.375}, {2.9, 0.65}, {3.2, 0.55}, {4.7, 0.83}},
    {{2.5, 0.82}, {3.0, 1.56}, {3.5, 2.96}, {0, 0}, {0, 0}},
    {{3.8, 0.40}, {3.6, 0.66}, {4.3, 0.88}, {4.9, 1.10}, {6.5, 1.33}},
    {{3.8, 0.58}, {4.0, 1.00}, {4.5, 1.78}, {8.0, 1.87}, {0, 0}},
    {{3.8, 0.58}, {4.0, 1.03}, {0, 0}, {6.5, 2.20}, {0, 0}}};
constexpr double LAUNCH = 2.5;

double kgm_us(int fmt, bool xf32, bool gated, int64_t maxM, int64_t M, int64_t N, int64_t K,
              int cus, int *shape)
{
    const Rate *const rates =
        RATES[!gated ? (xf32 ? 1 : 0) : fmt == QL_FMT_MXFP4 ? 2 : fmt == QL_FMT_Q4 ? 3 : 4];
    double best = 1e30;
    for (int s = 0; s < KGM_SHAPES; ++s) {
        const KgTile t = kgm_tile_shape(fmt, xf32, gated, maxM, s);
        if (!t.m)
            continue;
        const double wgs = (double)((M + t.m - 1) / t.m) * (double)((N + t.n - 1) / t.n);
        if (wgs * QL_MAX_GROUP > 4194303.0)  // (a launch has fewer than 2^32 threads)
            continue;
        const double r = wgs / cus, rounds = r <= 4.0 ? std::ceil(r) : r + 0.5;
        const double us = LAUNCH + rounds * (rates[s].fixed + (double)K / 256 * rates[s].per256);
        if (us < best) {
            best = us;
            *shape = s;
        }
    }
    return best;
}

RowsKernel choose_rows(int fmt, bool xf32, bool gated, int64_t maxM, int64_t M, int64_t N,
                       int64_t K, int cus, int *shape)
{
    *shape = 0;
    // few rows of short reductions: the kernel without stages starts faster (us there
    // / here: fp32 6144 x 1536 at 1 row 8.1 / 10.3, at 32 18.4 / 14.9; pairs at one
    // row, MXFP4 4096 x 1536 5.5 / 6.9, 1536 x 6144 12.7 / 11.3, q4 1024 x 1024 6.0 /
    // 6.6, 6144 x 1536 11.1 / 8.2)
    const bool few = M <= 16 && (gated ? K <= (fmt == QL_FMT_MXFP4 ? 2048 : 1024) : xf32);
    if (few || !kgm_takes(K))
        return ROWS_ANY;
    const double us = kgm_us(fmt, xf32, gated, maxM, M, N, K, cus, shape);
    int rows = 0;
    if (tile_takes(K) && tile_us(fmt, xf32, gated, M, N, K, cus, &rows) < us) {
        *shape = rows;
        return ROWS_TILE;
    }
    return us < 1e30 ? ROWS_KGM : ROWS_ANY;
}

hipError_t launch_qgemm_kgm(int fmt, bool xf32, RowsGroup &g, hipStream_t stream)
{
    const bool gated = g.d[0].codes[1] != nullptr;
    const int maxM = g.maxM;
    int64_t total = 0;
    for (int i = 0; i <= QL_MAX_GROUP; ++i) {
        g.begin[i] = (int)total;
        if (i < g.n) {
            const KgTile t = kgm_tile_shape(fmt, xf32, gated, maxM, g.d[i].shape);
            total += ((int64_t)g.d[i].M + t.m - 1) / t.m * (((int64_t)g.d[i].N + t.n - 1) / t.n);
        }
    }
    with_shapes(fmt, xf32, gated, maxM, [&](auto s) {
        hipLaunchKernelGGL(qgemm_kgm_kernel<decltype(s)>, dim3((unsigned)total), dim3(NT), 0,
                           stream, g);
        return 0;
    });
    return hipGetLastError();
}

}  // namespace qlk
