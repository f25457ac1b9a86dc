// Products with MXFP4 weights, and gated pairs of projections in any of the
// quantized formats, at many rows (bf16 activations):
//
//   P[m][n] = sum_k X[m][k] W[n][k],   W = c * s
//
// Weights become bf16 in registers: MXFP4 values are exact there (one
// instruction turns two codes and the block's scale into two bf16), a q4 / int8
// weight enters as the sum of two bf16 (off by at most 2^-18 of itself).  fp32
// activations come as three bf16 planes (launch_split3), one after the other
// along the reduction.
//
// Matrix instruction v_mfma_f32_32x32x16_bf16: lane l holds A[l % 32][8 (l / 32)
// + e] and B[8 (l / 32) + e][l % 32]; accumulator register r of lane l is
// D[8 (r / 4) + 4 (l / 32) + r % 4][l % 32].  Within a 64-k step, slot e of lane
// half g in chunk q holds k = 32 g + 8 q + e: a lane's weights over the step are
// one scale block, one 16-byte LDS read (int8: two).
//
// Tile: 4 wavefronts compute 128 rows x 256 weight rows, each a strip of 64
// weight rows (4 x 2 MFMA tiles): every converted weight feeds 4 MFMAs.  Of a
// gated pair the strip is 32 rows of the gate and the same 32 of the up
// projection, so both projections of an output meet in one lane and the
// activation and the product happen on the accumulators.
//
// Memory pipeline: direct-to-LDS loads of activations, codes and scales into a
// ring of stages of 64 k (three; int8 two), chunks of 16 bytes XOR-swizzled;
// one barrier per stage, at which a wavefront's own loads of the stage have
// landed and the slot two stages back is free.  Two workgroups per CU.  Scales:
// where a row's allow it, 16 bytes (MXFP4: of eight steps, fp16: of four) into
// one slot that every wavefront copies to registers at the group's start, so that
// it can be refilled behind them; otherwise dwords, one or two steps at a time (a
// memory request per row each: as many as the codes).
#include <algorithm>

#include "dma.h"
#include "internal.h"
#include "mx.h"
#include "strip.h"

namespace qlk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int BM = 128, BN = 256, MS = 4, NS = 2;
constexpr int GROUP_M = 4;

template <int FMT>
struct Geo {
    static constexpr int CROW = FMT == QL_FMT_INT8 ? 64 : 32;  // code bytes per row per step
    static constexpr int CCH = CROW / 16;
    static constexpr int XBYTES = BM * 128, CBYTES = BN * CROW, SBYTES = BN * 4;
    static constexpr int SSTEPS = FMT == QL_FMT_MXFP4 ? 2 : 1;  // steps of a scale dword
    static constexpr int STAGE = XBYTES + CBYTES;
    static constexpr int SLDS = 4 * SBYTES;  // a slot of 16 bytes per row, or a ring of 3 dwords
    static constexpr int NST = 2 * (3 * STAGE + SLDS) <= 160 * 1024 ? 3 : 2;
    static constexpr int LDS = NST * STAGE + SLDS;
    static constexpr int XLOADS = XBYTES / 16 / THREADS, CLOADS = CBYTES / 16 / THREADS;
    static constexpr int LOADS = XLOADS + CLOADS;
    static constexpr int PLANES = FMT == QL_FMT_MXFP4 ? 1 : 2;
    static_assert(2 * LDS <= 160 * 1024, "two workgroups per CU");
    static_assert(BN == THREADS, "one scale dword per thread");
};

// physical 16-byte chunk = logical ^ swizzle(row), so that the 16 lanes that one
// cycle of a 16-byte LDS read serves (rows 0-3, 12-15, 20-27, or the others of 32)
// meet distinct banks
__device__ inline int xswz(int row) { return (row & 7) ^ ((row >> 3) & 1); }
template <int FMT>
__device__ inline int cswz(int row)
{
    return FMT == QL_FMT_INT8 ? ((row >> 2) & 3) ^ ((row >> 4) & 1) * 3 : ((row >> 2) ^ (row >> 3)) & 1;
}

// weight row of the tile's row r (see the header): gated pairs alternate 32
// rows of the gate and 32 of the up projection
template <bool GATED>
__device__ inline int tile_row(int r)
{
    return GATED ? (r >> 6) * 32 + (r & 31) : r;
}

// SWIDE: scales 16 bytes at a time.  EPI: an epilogue beyond the output's type.
template <int FMT, bool GATED, bool SWIDE, bool EPI>
__global__ __launch_bounds__(THREADS, 2) void qgemm_tile_kernel(const TileArgs a)
{
    using G = Geo<FMT>;
    constexpr int NST = G::NST, P = G::PLANES;
    constexpr int COLS = GATED ? BN / 2 : BN;  // output columns of a tile
    constexpr int SG = SWIDE ? 4 * G::SSTEPS : 2;  // steps of a scale group
    __shared__ __align__(16) uint8_t ring[G::LDS];
    uint8_t *const sring = ring + NST * G::STAGE;
    const int M = a.M, N = a.N, K = a.K, nb = K >> 5;
    const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + COLS - 1) / COLS;
    // each XCD takes a contiguous range of the tiles, in groups of 4 row tiles
    // walked row tile fastest; the parts of a tile are adjacent
    const int p = (int)blockIdx.x, grid = (int)gridDim.x;
    const int gq = grid >> 3, gr = grid & 7, xcd = p & 7, idx = p >> 3;
    const int local = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int part = local % a.parts, tile = local / a.parts;
    const int gid = tile / (GROUP_M * tiles_n), within = tile - gid * (GROUP_M * tiles_n);
    const int gsz = min(tiles_m - gid * GROUP_M, GROUP_M);
    const int m0 = (gid * GROUP_M + within % gsz) * BM, n0 = within / gsz * COLS;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, g = lane >> 5;

    const int plane_steps = K >> 6, all_steps = plane_steps * a.planes;
    // parts of whole scale groups (a plane is some, too)
    const int per = ((all_steps + a.parts - 1) / a.parts + SG - 1) / SG * SG;
    const int s0 = part * per, ns = max(0, min(all_steps, s0 + per) - s0);

    // per-lane offsets within the tile; rows past the end repeat the last one
    uint32_t xoff[G::XLOADS];
    const uint8_t *cptr[G::CLOADS];
    uint32_t coff[G::CLOADS];
#pragma unroll
    for (int r = 0; r < G::XLOADS; ++r) {
        const int slot = r * THREADS + tid, row = slot >> 3, lc = (slot & 7) ^ xswz(row);
        xoff[r] = (uint32_t)((min(m0 + row, M - 1) - m0) * K * 2 + lc * 16);
    }
    const uint8_t *const cbase[2] = {a.codes[0], a.codes[GATED ? 1 : 0]};
    const uint8_t *const sbase[2] = {static_cast<const uint8_t *>(a.scales[0]),
                                     static_cast<const uint8_t *>(a.scales[GATED ? 1 : 0])};
    const int crow = K / 32 * (G::CROW / 2), srow = nb * (FMT == QL_FMT_MXFP4 ? 1 : 2);
    // (a wavefront's chunks of one load lie in rows of one projection: 64 lanes
    // cover 32 rows of 2 chunks, or 16 of 4)
#pragma unroll
    for (int r = 0; r < G::CLOADS; ++r) {
        const int slot = r * THREADS + tid, row = slot / G::CCH, lc = (slot % G::CCH) ^ cswz<FMT>(row);
        const int n = min(n0 + tile_row<GATED>(row), N - 1) - n0;
        const int up = GATED ? __builtin_amdgcn_readfirstlane((row >> 5) & 1) : 0;
        cptr[r] = cbase[up] + (int64_t)n0 * crow;
        coff[r] = (uint32_t)(n * crow + lc * 16);
    }
    // a wavefront's 64 scale rows: of a gated pair, half of each projection
    const uint8_t *const sp = sbase[GATED ? (tid >> 5) & 1 : 0] +
                              (int64_t)min(n0 + tile_row<GATED>(tid), N - 1) * srow;

    const uint8_t *const xb = static_cast<const uint8_t *>(a.X) + (int64_t)m0 * K * 2;
    auto issue = [&](int t) {  // step s0 + t into its slots
        const int s = s0 + t, plane = s / plane_steps, ks = s - plane * plane_steps;
        uint8_t *const st = ring + t % NST * G::STAGE;
        const uint32_t base = dma_lds(st);
        const uint8_t *const x = xb + plane * a.plane_bytes + (int64_t)ks * 128;
#pragma unroll
        for (int r = 0; r < G::XLOADS; ++r)
            dma_load16(x, xoff[r], base + (r * THREADS + wave * 64) * 16);
#pragma unroll
        for (int r = 0; r < G::CLOADS; ++r)
            dma_load16(cptr[r] + (int64_t)ks * G::CROW, coff[r],
                       base + G::XBYTES + (r * THREADS + wave * 64) * 16);
        if (!SWIDE && (G::SSTEPS == 1 || t % 2 == 0))
            dma_load4_at(sp + (int64_t)(ks / G::SSTEPS) * 4,
                         dma_lds(sring + t / G::SSTEPS % 3 * G::SBYTES) + wave * 256);
    };

    auto issue_scales = [&](int t) {  // of the group from step s0 + t (or the last one)
        const int s = s0 + min(t, ns - SG), ks = s - s / plane_steps * plane_steps;
        dma_load16_at(sp + (int64_t)(ks / G::SSTEPS) * 4, dma_lds(sring) + wave * 1024);
    };

    f32x16 acc[MS][NS];
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.f;

    if (SWIDE && ns > 0)
        issue_scales(0);
#pragma unroll
    for (int t = 0; t < NST - 1; ++t)
        if (t < ns)
            issue(t);
    u32x4 sgrp[NS];  // SWIDE: the group's scales of this lane's rows
    auto step = [&](int t, auto uc) {
        constexpr int U = decltype(uc)::value, ODD = U & 1;  // t % SG
        // loads land in order: with three stages the next one's may be in flight,
        // and what was issued with it: a scale dword with an even step, the next
        // group's scales behind the second step's barrier
        constexpr int EXTRA = SWIDE ? U == 2 : G::SSTEPS == 1 || ODD;
        if (NST == 3 && t + 1 < ns)
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(G::LOADS + EXTRA));
        else
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(0));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        if (t + NST - 1 < ns)
            issue(t + NST - 1);
        if constexpr (SWIDE && U == 1)
            issue_scales(t - 1 + SG);
        const uint8_t *const st = ring + t % NST * G::STAGE;
        uint32_t raw[NS][4 * G::CCH / 2];
        float sc[NS];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int row = wave * 64 + 32 * j + l32;
            uint32_t d;
            if constexpr (SWIDE) {
                if constexpr (U == 0)
                    sgrp[j] = *reinterpret_cast<const u32x4 *>(sring + row * 16);
                d = sgrp[j][U / G::SSTEPS];
            } else {
                d = *reinterpret_cast<const uint32_t *>(sring + t / G::SSTEPS % 3 * G::SBYTES +
                                                        row * 4);
            }
            if constexpr (FMT == QL_FMT_MXFP4)
                sc[j] = mx_scale(d >> (16 * ODD + 8 * g) & 255u);
            else
                sc[j] = (float)__builtin_bit_cast(_Float16, (uint16_t)(d >> (16 * g)));
#pragma unroll
            for (int h = 0; h < G::CCH / 2; ++h) {
                const int lc = g * (G::CCH / 2) + h;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(
                    st + G::XBYTES + (row * G::CCH + (lc ^ cswz<FMT>(row))) * 16);
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    raw[j][4 * h + w] = v[w];
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x4 xa[MS], wb[NS][P];
#pragma unroll
            for (int i = 0; i < MS; ++i) {
                const int row = 32 * i + l32;
                xa[i] = *reinterpret_cast<const u32x4 *>(
                    st + (row * 8 + ((4 * g + q) ^ xswz(row))) * 16);
            }
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                if constexpr (FMT == QL_FMT_MXFP4) {
                    wb[j][0] = mx_bf16x8(raw[j][q], sc[j]);
                } else {
                    float v[8];
                    if constexpr (FMT == QL_FMT_Q4)
                        q4_f32x8(raw[j][q], sc[j], v);
                    else
                        int8_f32x8(raw[j][2 * q], raw[j][2 * q + 1], sc[j], v);
                    split2(v, wb[j][0], wb[j][P - 1]);
                }
            }
#pragma unroll
            for (int v = P - 1; v >= 0; --v)
#pragma unroll
                for (int i = 0; i < MS; ++i)
#pragma unroll
                    for (int j = 0; j < NS; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(bf16x8, xa[i]),
                            __builtin_bit_cast(bf16x8, wb[j][v]), acc[i][j], 0, 0, 0);
        }
        pin_accumulators(acc);
    };
    // (ns is a multiple of SG: K % 128 == 0, and whole groups where SWIDE)
#pragma unroll 1
    for (int t = 0; t < ns; t += SG) {
        step(t, std::integral_constant<int, 0>{});
        step(t + 1, std::integral_constant<int, 1>{});
        if constexpr (SG >= 4) {
            step(t + 2, std::integral_constant<int, 2>{});
            step(t + 3, std::integral_constant<int, 3>{});
        }
        if constexpr (SG == 8) {
            step(t + 4, std::integral_constant<int, 4>{});
            step(t + 5, std::integral_constant<int, 5>{});
            step(t + 6, std::integral_constant<int, 6>{});
            step(t + 7, std::integral_constant<int, 7>{});
        }
    }
    __syncthreads();  // the ring is free: the 32 x 32 tiles turn through patches of it

    float *const patch = reinterpret_cast<float *>(ring) + wave * STRIP_PATCH;
    if constexpr (GATED) {
        strip_gated(a.gate, M, N, m0, n0 + wave * 32, patch, lane, acc);
    } else {
        const bool to_part = a.parts > 1;
        float *const Y = to_part ? a.part + (int64_t)part * M * N : a.Y;
        strip_store<EPI>(a.ep, Y, M, N, m0, n0 + wave * 64, patch, lane, acc,
                         epi_vec_ok(a.ep, Y, N), !to_part);
    }
}

// fp32 X as three bf16 planes [3][count], largest first: the first two by
// truncation, so that every remainder is exact
__global__ __launch_bounds__(256) void split3_kernel(const float *__restrict__ X, int64_t groups,
                                                     uint16_t *__restrict__ out, int64_t plane)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < groups;
         i += (int64_t)gridDim.x * 256) {
        float v[8];
        *reinterpret_cast<f32x4 *>(v) = reinterpret_cast<const f32x4 *>(X)[2 * i];
        *reinterpret_cast<f32x4 *>(v + 4) = reinterpret_cast<const f32x4 *>(X)[2 * i + 1];
        u32x4 p[3];
        split3(v, p);
#pragma unroll
        for (int q = 0; q < 3; ++q)
            reinterpret_cast<u32x4 *>(out + q * plane)[i] = p[q];
    }
}

}  // namespace

int64_t tile_tiles(int64_t M, int64_t N, bool gated)
{
    const int cols = gated ? BN / 2 : BN;
    return (M + BM - 1) / BM * ((N + cols - 1) / cols);
}

bool tile_takes(int64_t K, const void *scales0, const void *scales1)
{
    return K % 128 == 0 && K < ((int64_t)1 << 22) && ((uintptr_t)scales0 & 3) == 0 &&
           ((uintptr_t)scales1 & 3) == 0;
}

bool tile_wins(int fmt, bool xf32, bool gated, int64_t M, int64_t N, int64_t K, int cus)
{
    (void)fmt;
    (void)xf32;
    (void)K;
    return tile_tiles(M, N, gated) >= cus / 2;
}

hipError_t launch_split3(const float *X, int64_t count, uint16_t *planes, hipStream_t stream)
{
    const int64_t groups = count / 8;
    hipLaunchKernelGGL(split3_kernel, dim3((unsigned)std::min<int64_t>((groups + 255) / 256, 1 << 20)),
                       dim3(256), 0, stream, X, groups, planes, count);
    return hipGetLastError();
}

hipError_t launch_qgemm_tile(int fmt, const TileArgs &a, hipStream_t stream)
{
    const bool gated = a.codes[1] != nullptr;
    const dim3 grid((unsigned)(tile_tiles(a.M, a.N, gated) * a.parts)), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    // scales in 16-byte chunks: whole groups in a row, 16-byte aligned
    const bool swide = a.K % (fmt == QL_FMT_MXFP4 ? 512 : 256) == 0 &&
                       (((uintptr_t)a.scales[0] | (uintptr_t)a.scales[1]) & 15) == 0;
    auto with = [&](auto fmtc, auto gatedc, auto epic) {
        constexpr int F = decltype(fmtc)::value;
        constexpr bool GD = decltype(gatedc)::value, E = decltype(epic)::value;
        swide ? go(qgemm_tile_kernel<F, GD, true, E>) : go(qgemm_tile_kernel<F, GD, false, E>);
    };
    using Mx = std::integral_constant<int, QL_FMT_MXFP4>;
    if (!gated && !strip_plain(a.ep))
        with(Mx{}, std::false_type{}, std::true_type{});
    else if (!gated)
        with(Mx{}, std::false_type{}, std::false_type{});
    else if (fmt == QL_FMT_MXFP4)
        with(Mx{}, std::true_type{}, std::false_type{});
    else if (fmt == QL_FMT_Q4)
        with(std::integral_constant<int, QL_FMT_Q4>{}, std::true_type{}, std::false_type{});
    else
        with(std::integral_constant<int, QL_FMT_INT8>{}, std::true_type{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace qlk
