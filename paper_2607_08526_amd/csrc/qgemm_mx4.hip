// Products of MXFP4 activations with MXFP4 weights at many rows, on the 4-bit
// matrix cores:
//
//   P[m][n] = sum_b 2^(sx[m][b] + sw[n][b] - 254) sum_{k in b} x[m][k] w[n][k]
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes codes and scale bytes as they are: lane
// l holds the 32 codes (16 bytes, one block) of row l % 32 and block l / 32 of a
// 64-k chunk, and that block's scale in one byte of a register.
//
// Tile, pipeline and store as in the bf16 tiles (qgemm_tile.hip): 4 wavefronts
// compute 128 or 64 rows x 256 weight rows (strips of 64 weight rows), stages of 128
// k move directly to LDS through a ring of three, 16-byte chunks XOR-swizzled, one
// barrier per stage.  Scales of the tile's rows: where a row's allow it, 16
// bytes (four stages) into one slot that every wavefront copies to registers at
// the group's start, so that it can be refilled behind them; otherwise each by
// itself with its stage (more memory requests than the codes), a ring of two.  A
// stage that K leaves unfilled ends in zeros.  Two workgroups per CU.
//
// Bound: latency where tiles are few (a wavefront per SIMD: hence the 64-row tiles,
// which are twice as many), the stores and the residual at short reductions, and
// operand traffic from L2 at long ones: 4096 x 8192 x 8192 (2 M N K = 550 Gflop) 165 to
// 174 us, 3.2 to 3.3 PFLOP/s.  1290 rows x 6144 x 1536 with bias, GELU and an fp32
// residual 26.6 us, 24.4 Gflop and 70 MB (14 us of a copy).
#include <algorithm>
#include <cmath>

#include "dma.h"
#include "internal.h"
#include "mx.h"
#include "strip.h"

namespace qlk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int BN = 256, NS = 2;
constexpr int ROW = 64;  // code bytes per row and stage (128 k)

__device__ __align__(16) const uint32_t zeros[4] = {0, 0, 0, 0};

// physical 16-byte chunk = logical ^ swz(row): a cycle of a 16-byte read serves
// rows 0-3, 12-15, 20-27, or the others of 32, and meets distinct banks
__device__ inline int swz(int row) { return ((row >> 2) & 3) ^ ((row >> 4) & 1) * 3; }

__device__ inline i32x8 codes8(u32x4 v)
{
    return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}

// SWIDE: scales 16 bytes at a time.  EPI: an epilogue beyond the output's type.
// MS: blocks of 32 rows of the tile.
template <int MS, bool SWIDE, bool EPI>
__global__ __launch_bounds__(THREADS, 2) void qgemm_mx4_kernel(const Mx4Args a)
{
    constexpr int BM = 32 * MS, GROUP_M = 16 / MS;
    constexpr int XBYTES = BM * ROW, WBYTES = BN * ROW, STAGE = XBYTES + WBYTES;
    constexpr int SROWS = BM + BN, SLDS = SROWS * 16;  // scales: 16 bytes, or 4 blocks' dwords
    constexpr int XLOADS = XBYTES / 16 / THREADS, WLOADS = WBYTES / 16 / THREADS;
    static_assert(2 * (3 * STAGE + SLDS) <= 160 * 1024 && 4 * (STAGE + SLDS) <= 160 * 1024,
                  "two workgroups per CU");
    constexpr int SG = SWIDE ? 4 : 1, NST = SWIDE ? 3 : 2;  // stages of a scale group, of the ring
    __shared__ __align__(16) uint8_t ring[NST * STAGE + (SWIDE ? 1 : NST) * SLDS];
    uint8_t *const sring = ring + NST * STAGE;
    const int M = a.M, N = a.N, nb = a.K >> 5;
    const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN;
    const int p = (int)blockIdx.x, grid = (int)gridDim.x;
    const int gq = grid >> 3, gr = grid & 7, xcd = p & 7, idx = p >> 3;
    const int tile = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int gid = tile / (GROUP_M * tiles_n), within = tile - gid * (GROUP_M * tiles_n);
    const int gsz = min(tiles_m - gid * GROUP_M, GROUP_M);
    const int m0 = (gid * GROUP_M + within % gsz) * BM, n0 = within / gsz * BN;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int ns = (nb + 3) >> 2;

    // per-lane offsets within the tile; rows past the end repeat the last one
    const int krow = nb * 16;
    uint32_t xoff[XLOADS], woff[WLOADS];
#pragma unroll
    for (int r = 0; r < XLOADS; ++r) {
        const int slot = r * THREADS + tid, row = slot >> 2, lc = (slot & 3) ^ swz(row);
        xoff[r] = (uint32_t)((min(m0 + row, M - 1) - m0) * krow + lc * 16);
    }
#pragma unroll
    for (int r = 0; r < WLOADS; ++r) {
        const int slot = r * THREADS + tid, row = slot >> 2, lc = (slot & 3) ^ swz(row);
        woff[r] = (uint32_t)((min(n0 + row, N - 1) - n0) * krow + lc * 16);
    }
    const uint32_t wsoff = (uint32_t)((min(n0 + tid, N - 1) - n0) * nb);
    const uint32_t xsoff = (uint32_t)((min(m0 + tid % BM, M - 1) - m0) * nb);
    const uint8_t *const xb = a.qx + (int64_t)m0 * krow, *const wb = a.codes + (int64_t)n0 * krow;
    const uint8_t *const xs = a.sx + (int64_t)m0 * nb, *const ws = a.scales + (int64_t)n0 * nb;
    // scales of the group that stage s starts: rows of X, then of W (not SWIDE: four
    // of them, one for each block; past K the row's last).  (X's by the first XH
    // wavefronts; SWIDE the others repeat them, so that every wavefront counts the
    // same loads, otherwise they take other blocks.)
    constexpr int XH = BM / 64;
    auto issue_scales = [&](int s) {
        if constexpr (SWIDE) {
            const uint32_t base = dma_lds(sring);
            dma_load16(ws + (int64_t)s * 4, wsoff, base + (BM + wave * 64) * 16);
            dma_load16(xs + (int64_t)s * 4, xsoff, base + wave % XH * 64 * 16);
        } else {
            const uint32_t base = dma_lds(sring + s % NST * SLDS);
#pragma unroll
            for (int h = 0; h < 4; ++h)
                dma_load_small_at<1>(ws + wsoff + min(4 * s + h, nb - 1),
                                     base + h * (SROWS * 4) + (BM + wave * 64) * 4);
#pragma unroll
            for (int h = 0; h < XH; ++h) {
                const int b = (4 * h + wave) / XH;
                dma_load_small_at<1>(xs + xsoff + min(4 * s + b, nb - 1),
                                     base + b * (SROWS * 4) + wave % XH * 64 * 4);
            }
        }
    };
    auto issue = [&](int s) {
        const uint32_t base = dma_lds(ring + s % NST * STAGE) + wave * 1024;
        const uint8_t *const x = xb + (int64_t)s * ROW, *const w = wb + (int64_t)s * ROW;
        if (SWIDE || 4 * s + 4 <= nb) {
#pragma unroll
            for (int r = 0; r < XLOADS; ++r)
                dma_load16(x, xoff[r], base + r * THREADS * 16);
#pragma unroll
            for (int r = 0; r < WLOADS; ++r)
                dma_load16(w, woff[r], base + XBYTES + r * THREADS * 16);
        } else {
            // (a chunk is a block)
            auto at = [&](const uint8_t *p, uint32_t off, int i) {
                return 4 * s + ((i & 3) ^ swz(i >> 2)) < nb ? p + off : (const uint8_t *)zeros;
            };
#pragma unroll
            for (int r = 0; r < XLOADS; ++r)
                dma_load16_at(at(x, xoff[r], r * THREADS + tid), base + r * THREADS * 16);
#pragma unroll
            for (int r = 0; r < WLOADS; ++r)
                dma_load16_at(at(w, woff[r], r * THREADS + tid), base + XBYTES + r * THREADS * 16);
        }
        if constexpr (!SWIDE)
            issue_scales(s);
    };
    constexpr int LOADS = XLOADS + WLOADS + (SWIDE ? 0 : 4 + XH);

    f32x16 acc[MS][NS];
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.f;

    if constexpr (SWIDE)
        issue_scales(0);
    issue(0);
    if (NST == 3 && ns > 1)
        issue(1);
    u32x4 ga[MS], gb[NS];  // SWIDE: the group's scales of this lane's rows
    auto step = [&](int s, auto uc) {
        constexpr int U = decltype(uc)::value;  // s % SG
        // loads land in order: the next stage's may be in flight, and the next
        // group's scales, issued behind the second stage's barrier
        if (NST == 3 && s + 1 < ns)
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(LOADS + (SWIDE && U == 2 ? 2 : 0)));
        else
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(0));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        if (s + NST - 1 < ns)
            issue(s + NST - 1);
        if constexpr (SWIDE && U == 1)  // (the last group again at the end)
            issue_scales(min(s - 1 + SG, ns - SG));
        const uint8_t *const st = ring + s % NST * STAGE;
        const uint8_t *const ss = sring + (SWIDE ? 0 : s % NST * SLDS);
        uint32_t sa[MS], sb[NS];  // byte 2 q: this lane's block (2 q + g) of chunk q
        auto scale = [&](int row, u32x4 &grp) {
            if constexpr (SWIDE) {
                if constexpr (U == 0)
                    grp = *reinterpret_cast<const u32x4 *>(ss + row * 16);
                return grp[U] >> (8 * g);
            } else {
                const uint32_t *const d = reinterpret_cast<const uint32_t *>(ss) + g * SROWS + row;
                return d[0] | d[2 * SROWS] << 16;
            }
        };
#pragma unroll
        for (int i = 0; i < MS; ++i)
            sa[i] = scale(32 * i + l32, ga[i]);
#pragma unroll
        for (int j = 0; j < NS; ++j)
            sb[j] = scale(BM + wave * 64 + 32 * j + l32, gb[j]);
        auto chunk = [&](auto qc) {
            constexpr int q = decltype(qc)::value;
            u32x4 av[MS], bv[NS];
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                const int row = wave * 64 + 32 * j + l32;
                bv[j] = *reinterpret_cast<const u32x4 *>(st + XBYTES +
                                                         (row * 4 + ((2 * q + g) ^ swz(row))) * 16);
            }
#pragma unroll
            for (int i = 0; i < MS; ++i) {
                const int row = 32 * i + l32;
                av[i] = *reinterpret_cast<const u32x4 *>(st + (row * 4 + ((2 * q + g) ^ swz(row))) * 16);
            }
#pragma unroll
            for (int i = 0; i < MS; ++i)
#pragma unroll
                for (int j = 0; j < NS; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        codes8(av[i]), codes8(bv[j]), acc[i][j], 4, 4, 2 * q, (int)sa[i], 2 * q,
                        (int)sb[j]);
        };
        chunk(std::integral_constant<int, 0>{});
        chunk(std::integral_constant<int, 1>{});
        pin_accumulators(acc);
    };
#pragma unroll 1
    for (int s = 0; s < ns; s += SG) {
        step(s, std::integral_constant<int, 0>{});
        if constexpr (SWIDE) {
            step(s + 1, std::integral_constant<int, 1>{});
            step(s + 2, std::integral_constant<int, 2>{});
            step(s + 3, std::integral_constant<int, 3>{});
        }
    }
    __syncthreads();  // the ring is free: the 32 x 32 tiles turn through patches of it

    float *const patch = reinterpret_cast<float *>(ring) + wave * STRIP_PATCH;
    strip_store<EPI>(a.ep, a.Y, M, N, m0, n0 + wave * 64, patch, lane, acc,
                     epi_vec_ok(a.ep, a.Y, N), true);
}

}  // namespace

int64_t mx4_tiles(const Mx4Args &a, int rows)
{
    return ((int64_t)a.M + rows - 1) / rows * (((int64_t)a.N + BN - 1) / BN);
}

bool mx4_takes(const Mx4Args &a)
{
    return a.K < (1 << 22);
}

// Estimated us of tiles of 64 or 128 rows.  A stage of a tile that has a CU to itself
// takes 0.37 or 0.53 us (latency: rising where most CUs work), one of several on a CU
// 0.46 or 0.66; an epilogue 4 us, with an activation 8, per 128 rows of a tile.
// Measured, 64 / 128 rows without an epilogue: 6144 x 1536 at 256 rows 9.3 / 12.8, at
// 1290 16.2 / 18.9, at 2048 21.2 / 20.3; 1536 x 6144 at 1290 rows 24.0 / 31.8, at 4096
// 42.4 / 34.1; with bias, GELU and residual 6144 x 1536 at 1290 rows 26.6 / 34.2.
static double mx4_us(const Mx4Args &a, int rows, int cus)
{
    const double r = (double)mx4_tiles(a, rows) / cus, up = std::ceil(r);
    const double steps = std::ceil(a.K / 128.0), busy = r + 0.4 * (up - r);
    const double stage = rows == 64 ? (r <= 1.0 ? 0.36 + 0.05 * r : 0.46 * busy)
                                    : (r <= 1.0 ? 0.49 + 0.13 * r : 0.66 * busy);
    const double epi = strip_plain(a.ep) ? 0.0 : a.ep.act ? 8.0 : 4.0;
    return (rows == 64 ? 5.0 : 5.5) + steps * stage +
           epi * rows / 128 * std::max(1.0, std::min(r, 2.0));
}

int mx4_rows(const Mx4Args &a, int cus)
{
    return mx4_us(a, 64, cus) < mx4_us(a, 128, cus) ? 64 : 128;
}

// Against the few-row kernel: a 128-k step there takes 0.13 to 0.32 us by its row tile
// and 0.85 ns per workgroup.
bool mx4_wins(const Mx4Args &a, int cus)
{
    const double steps = std::ceil(a.K / 128.0);
    const int rows = a.M <= 16 ? 16 : a.M <= 32 ? 32 : 64;
    const double wgs = (double)((a.M + rows - 1) / rows) * ((a.N + 31) / 32);
    const double few = 4.5 + steps * ((rows == 16 ? 0.13 : rows == 32 ? 0.19 : 0.32) + 0.00085 * wgs);
    return std::min(mx4_us(a, 64, cus), mx4_us(a, 128, cus)) < few;
}

hipError_t launch_qgemm_mx4(const Mx4Args &a, hipStream_t stream)
{
    const int rows = mx4_rows(a, current_cus());
    const dim3 grid((unsigned)mx4_tiles(a, rows)), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    const bool epi = !strip_plain(a.ep);
    const bool swide = a.K % 512 == 0 && (((uintptr_t)a.sx | (uintptr_t)a.scales) & 15) == 0;
    auto with = [&](auto msc) {
        constexpr int MS = decltype(msc)::value;
        if (swide)
            epi ? go(qgemm_mx4_kernel<MS, true, true>) : go(qgemm_mx4_kernel<MS, true, false>);
        else
            epi ? go(qgemm_mx4_kernel<MS, false, true>) : go(qgemm_mx4_kernel<MS, false, false>);
    };
    rows == 64 ? with(std::integral_constant<int, 2>{}) : with(std::integral_constant<int, 4>{});
    return hipGetLastError();
}

}  // namespace qlk
