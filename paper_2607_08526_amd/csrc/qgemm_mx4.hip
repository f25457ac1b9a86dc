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
// compute 128 rows x 256 weight rows (strips of 64), stages of 128 k move
// directly to LDS through a ring of three, 16-byte chunks XOR-swizzled, one
// barrier per stage.  Scales of the tile's 384 rows: where a row's allow it, 16
// bytes (four stages) into one slot that every wavefront copies to registers at
// the group's start, so that it can be refilled behind them; otherwise a dword
// with each stage (as many memory requests as the codes).  Two workgroups per CU.
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
constexpr int BM = 128, BN = 256, MS = 4, NS = 2;
constexpr int GROUP_M = 4;
constexpr int ROW = 64;  // code bytes per row and stage (128 k)
constexpr int XBYTES = BM * ROW, WBYTES = BN * ROW;
constexpr int STAGE = XBYTES + WBYTES, NST = 3;
constexpr int SROWS = BM + BN, SLDS = SROWS * 16;  // scales: a slot of 16 bytes, or 3 of 4
constexpr int XLOADS = XBYTES / 16 / THREADS, WLOADS = WBYTES / 16 / THREADS;
static_assert(2 * (NST * STAGE + SLDS) <= 160 * 1024, "two workgroups per CU");

// physical 16-byte chunk = logical ^ swz(row): a cycle of a 16-byte read serves
// rows 0-3, 12-15, 20-27, or the others of 32, and meets distinct banks
__device__ inline int swz(int row) { return ((row >> 2) & 3) ^ ((row >> 4) & 1) * 3; }

__device__ inline i32x8 codes8(u32x4 v)
{
    return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}

// SWIDE: scales 16 bytes at a time.  EPI: an epilogue beyond the output's type.
template <bool SWIDE, bool EPI>
__global__ __launch_bounds__(THREADS, 2) void qgemm_mx4_kernel(const Mx4Args a)
{
    constexpr int SG = SWIDE ? 4 : 1, SB = SWIDE ? 16 : 4;  // stages, bytes of a scale group
    __shared__ __align__(16) uint8_t ring[NST * STAGE + SLDS];
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
    const int ns = a.K >> 7;

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
    const uint32_t xsoff = (uint32_t)((min(m0 + (tid & 127), M - 1) - m0) * nb);
    const uint8_t *const xb = a.qx + (int64_t)m0 * krow, *const wb = a.codes + (int64_t)n0 * krow;
    const uint8_t *const xs = a.sx + (int64_t)m0 * nb, *const ws = a.scales + (int64_t)n0 * nb;
    // scales of the group that stage s starts: rows of X, then of W.  (X's by the
    // first two wavefronts; the others repeat them, so that every wavefront counts
    // the same loads)
    auto issue_scales = [&](int s) {
        const uint32_t base = dma_lds(sring + (SWIDE ? 0 : s % 3) * (SROWS * 4));
        const uint32_t xl = base + (wave & 1) * 64 * SB, wl = base + (BM + wave * 64) * SB;
        if constexpr (SWIDE) {
            dma_load16(ws + (int64_t)s * 4, wsoff, wl);
            dma_load16(xs + (int64_t)s * 4, xsoff, xl);
        } else {
            dma_load4(ws + (int64_t)s * 4, wsoff, wl);
            dma_load4(xs + (int64_t)s * 4, xsoff, xl);
        }
    };
    auto issue = [&](int s) {
        const uint32_t base = dma_lds(ring + s % NST * STAGE);
#pragma unroll
        for (int r = 0; r < XLOADS; ++r)
            dma_load16(xb + (int64_t)s * ROW, xoff[r], base + (r * THREADS + wave * 64) * 16);
#pragma unroll
        for (int r = 0; r < WLOADS; ++r)
            dma_load16(wb + (int64_t)s * ROW, woff[r],
                       base + XBYTES + (r * THREADS + wave * 64) * 16);
        if constexpr (!SWIDE)
            issue_scales(s);
    };
    constexpr int LOADS = XLOADS + WLOADS + (SWIDE ? 0 : 2);

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
    if (ns > 1)
        issue(1);
    u32x4 ga[MS], gb[NS];  // SWIDE: the group's scales of this lane's rows
    auto step = [&](int s, auto uc) {
        constexpr int U = decltype(uc)::value;  // s % SG
        // loads land in order: the next stage's may be in flight, and the next
        // group's scales, issued behind the second stage's barrier
        if (s + 1 < ns)
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(LOADS + (SWIDE && U == 2 ? 2 : 0)));
        else
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(0));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        if (s + 2 < ns)
            issue(s + 2);
        if constexpr (SWIDE && U == 1)  // (the last group again at the end)
            issue_scales(min(s - 1 + SG, ns - SG));
        const uint8_t *const st = ring + s % NST * STAGE;
        const uint8_t *const ss = sring + (SWIDE ? 0 : s % 3) * (SROWS * 4);
        uint32_t sa[MS], sb[NS];  // byte 2 q: this lane's block of chunk q
        auto scale = [&](int row, u32x4 &grp) {
            if constexpr (SWIDE) {
                if constexpr (U == 0)
                    grp = *reinterpret_cast<const u32x4 *>(ss + row * 16);
                return grp[U] >> (8 * g);
            } else {
                return *reinterpret_cast<const uint32_t *>(ss + row * 4) >> (8 * g);
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

static int64_t mx4_tiles(const Mx4Args &a)
{
    return ((int64_t)a.M + BM - 1) / BM * (((int64_t)a.N + BN - 1) / BN);
}

bool mx4_takes(const Mx4Args &a)
{
    return a.K % 128 == 0 && a.K < (1 << 22) && ((uintptr_t)a.sx & 3) == 0 &&
           ((uintptr_t)a.scales & 3) == 0;
}

// Estimated us: a stage of a tile takes 0.49 us while few CUs work, 0.62 when all
// do, two on a CU 0.66 each; a 128-k step of the few-row kernel 0.13 to 0.32 us by
// its row tile and 0.85 ns per workgroup (6144 x 1536, tiles / few rows: 128 rows
// 11.5 / 10.0, 256 rows 11.4 / 13.9, 1024 rows 12.8 / 41.7; 1536 x 6144: 256 rows
// 29.1 / 19.9, 1024 rows 29.7 / 51.5).
bool mx4_wins(const Mx4Args &a, int cus)
{
    const double r = (double)mx4_tiles(a) / cus, up = std::ceil(r), steps = (double)(a.K / 128);
    const double tile = 5.5 + steps * (r <= 1.0 ? 0.49 + 0.13 * r : 0.66 * (r + 0.4 * (up - r)));
    const int rows = a.M <= 16 ? 16 : a.M <= 32 ? 32 : 64;
    const double wgs = (double)((a.M + rows - 1) / rows) * ((a.N + 31) / 32);
    const double few = 4.5 + steps * ((rows == 16 ? 0.13 : rows == 32 ? 0.19 : 0.32) + 0.00085 * wgs);
    return tile < few;
}

hipError_t launch_qgemm_mx4(const Mx4Args &a, hipStream_t stream)
{
    const dim3 grid((unsigned)mx4_tiles(a)), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    const bool epi = !strip_plain(a.ep);
    if (a.K % 512 == 0 && (((uintptr_t)a.sx | (uintptr_t)a.scales) & 15) == 0)
        epi ? go(qgemm_mx4_kernel<true, true>) : go(qgemm_mx4_kernel<true, false>);
    else
        epi ? go(qgemm_mx4_kernel<false, true>) : go(qgemm_mx4_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace qlk
