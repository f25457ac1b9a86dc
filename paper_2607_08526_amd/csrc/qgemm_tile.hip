// Products with MXFP4 weights, and gated pairs of projections in any of the
// quantized formats, at many rows (bf16 activations):
//
//   P[m][n] = sum_k X[m][k] W[n][k],   W = c * s
//
// Weights become bf16 in registers: MXFP4 values are exact there (one
// instruction turns two codes and the block's scale into two bf16), a q4 / int8
// weight enters as the sum of two bf16 (off by at most 2^-22 / 2^-16 of itself: mx.h).  fp32
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
// weight rows (4 x 2 MFMA tiles): every converted weight feeds 4 MFMAs; or 64 rows,
// where tiles are few: twice as many wavefronts hide the latency that bounds them.  Of a
// gated pair the strip is 32 rows of the gate and the same 32 of the up
// projection, so both projections of an output meet in one lane and the
// activation and the product happen on the accumulators.
//
// Memory pipeline: direct-to-LDS loads of activations, codes and scales into a
// ring of stages of 64 k (three; int8 two), chunks of 16 bytes XOR-swizzled.  The
// step's barrier sits before its last 16-k chunk: by then a stage is in registers
// and its slot refilled at once, while that chunk runs and prepares the next
// stage's first one.  Behind every MFMA goes a share of the next chunk's LDS reads
// and conversions.  Two workgroups per CU.  Scales: where a row's allow it, 16 bytes
// (MXFP4: of eight steps, fp16: of four) into one slot that every wavefront copies
// to registers at the group's start, so that it can be refilled behind them;
// otherwise each by itself with its step (a memory request each: as many as the
// codes).  Steps that K leaves unfilled, and those that fill up the loop's rounds,
// come from a page of zeros.
//
// Bound: the issue of matrix and vector instructions.  While a CU holds a workgroup its
// matrix cores are busy 0.53 (products) to 0.62 (pairs) of the cycles; wavefronts wait
// 0.45 of theirs for an instruction's unit, 0.11 to 0.23 for data or a barrier.  Then the
// clock (1.6 GHz of 2.4 in a run of 32768 rows), and at the end of a tile, where every CU
// is there at once, the VALU of the activation and the stores.  2048 rows x 8192 x 2048
// with GELU, bf16 output: 65 to 67 us, 1.03 to 1.06 PFLOP/s (a library product of 8192^3
// bf16 1.5); gated pair 2048 x 5504 x 2048 with SiLU: 80 to 84 us, 1.10 to 1.16 PFLOP/s,
// 688 tiles on 512 places; of q4 174 and of int8 170 us (two planes: twice the matrix
// instructions).  The 128-row tiles of int8 spill 28 registers (67 with scales one by
// one), of q4 47 with scales one by one.
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
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int BN = 256, NS = 2;

// MS: blocks of 32 rows of the tile.
template <int FMT, int MS>
struct Geo {
    static constexpr int BM = 32 * MS;
    static constexpr int CROW = FMT == QL_FMT_INT8 ? 64 : 32;  // code bytes per row per step
    static constexpr int CCH = CROW / 16;
    static constexpr int XBYTES = BM * 128, CBYTES = BN * CROW;
    static constexpr int SB = FMT == QL_FMT_MXFP4 ? 1 : 2;      // bytes of a scale
    static constexpr int SSTEPS = FMT == QL_FMT_MXFP4 ? 2 : 1;  // steps of a dword of scales
    static constexpr int STAGE = XBYTES + CBYTES;
    static constexpr int SSTEP = 2 * BN * 4;  // a step's scales, a dword each
    static constexpr int SLDS = 3 * SSTEP;    // (or a slot of 16 bytes per row)
    static constexpr int NST = 2 * (3 * STAGE + SLDS) <= 160 * 1024 ? 3 : 2;
    static constexpr int LDS = NST * STAGE + SLDS;
    static constexpr int XLOADS = XBYTES / 16 / THREADS, CLOADS = CBYTES / 16 / THREADS;
    static constexpr int LOADS = XLOADS + CLOADS;
    static constexpr int PLANES = FMT == QL_FMT_MXFP4 ? 1 : 2;
    static_assert(2 * LDS <= 160 * 1024, "two workgroups per CU");
    static_assert(BN == THREADS, "one scale dword per thread");
};

__device__ __align__(16) const uint32_t zeros[4] = {0, 0, 0, 0};

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

// What a lane needs of a tile, fixed for the whole reduction, and how far the
// loads have come.
template <int FMT, int MS, bool SWIDE>
struct Ctx {
    uint8_t *ring, *sring;
    uint32_t xoff[Geo<FMT, MS>::XLOADS], coff[Geo<FMT, MS>::CLOADS];
    const uint8_t *cptr[Geo<FMT, MS>::CLOADS];  // wave-uniform
    const uint8_t *x;                       // of the next stage to load
    const uint8_t *sp;                      // this thread's scale row
    int64_t plane_skip;                     // from one plane's end to the next one
    int plane_steps, planes;                // steps of a plane; planes from this one on
    int nb, ik, sk;                         // blocks of a row; next stage, next scale group
    int wave, lane;
};

// Operands carried from one 16-k chunk to the next, across stages too: the
// step's raw codes and scales, and the fragments of the chunk about to be
// multiplied.
template <int FMT, int MS>
struct Ops {
    uint32_t raw[NS][4 * Geo<FMT, MS>::CCH / 2];
    float sc[NS];
    u32x4 grp[NS];  // a scale group's dwords (not SWIDE: one)
    u32x4 a[MS], b[NS][Geo<FMT, MS>::PLANES];
};

// Loads of step t, the next stage, into its slot, and where scales are not SWIDE
// the step's (of blocks past K: the row's last).
template <int FMT, int MS, bool SWIDE>
__device__ inline void issue(Ctx<FMT, MS, SWIDE> &c, int t, int slot)
{
    using G = Geo<FMT, MS>;
    const uint32_t base = dma_lds(c.ring + slot * G::STAGE) + c.wave * 1024;
    const int left = c.nb - 2 * c.ik;  // blocks from this step on
    if (SWIDE || left >= 2) {
#pragma unroll
        for (int r = 0; r < G::XLOADS; ++r)
            dma_load16(c.x, c.xoff[r], base + r * THREADS * 16);
#pragma unroll
        for (int r = 0; r < G::CLOADS; ++r)
            dma_load16(c.cptr[r] + c.ik * G::CROW, c.coff[r], base + G::XBYTES + r * THREADS * 16);
    } else {
        const int tid = c.wave * 64 + c.lane;
#pragma unroll
        for (int r = 0; r < G::XLOADS; ++r) {
            const int i = r * THREADS + tid, lc = (i & 7) ^ xswz(i >> 3);
            dma_load16_at(lc / 4 < left ? c.x + c.xoff[r] : (const uint8_t *)zeros,
                          base + r * THREADS * 16);
        }
#pragma unroll
        for (int r = 0; r < G::CLOADS; ++r) {
            const int i = r * THREADS + tid, lc = (i % G::CCH) ^ cswz<FMT>(i / G::CCH);
            dma_load16_at(lc / (G::CCH / 2) < left ? c.cptr[r] + c.ik * G::CROW + c.coff[r]
                                                   : (const uint8_t *)zeros,
                          base + G::XBYTES + r * THREADS * 16);
        }
    }
    if constexpr (!SWIDE) {
        const uint32_t to = dma_lds(c.sring + t % 3 * G::SSTEP) + c.wave * 256;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            dma_load_small_at<G::SB>(c.sp + min(2 * c.ik + h, c.nb - 1) * G::SB, to + h * BN * 4);
    }
    c.x += 128;
    if (++c.ik == c.plane_steps && c.planes > 1) {
        --c.planes;
        c.ik = 0;
        c.x += c.plane_skip;
    }
}

// SWIDE: 16 bytes per row, the next scale group (past the last: a group of the
// row that is not used)
template <int FMT, int MS, bool SWIDE>
__device__ inline void issue_scales(Ctx<FMT, MS, SWIDE> &c)
{
    dma_load16_at(c.sp + (c.sk / Geo<FMT, MS>::SSTEPS) * 4, dma_lds(c.sring) + c.wave * 1024);
    c.sk += 4 * Geo<FMT, MS>::SSTEPS;
    if (c.sk == c.plane_steps)
        c.sk = 0;
}

__device__ inline u32x4 read_x(const uint8_t *st, int lane, int q, int i)
{
    const int row = 32 * i + (lane & 31);
    return *reinterpret_cast<const u32x4 *>(st + (row * 8 + ((4 * (lane >> 5) + q) ^ xswz(row))) *
                                                     16);
}

// codes and scale of step t (from stage st) for fragment j; U = t % 4
template <int FMT, int MS, bool SWIDE, int U>
__device__ inline void read_weights(const Ctx<FMT, MS, SWIDE> &c, const uint8_t *st, int t, int j,
                                    Ops<FMT, MS> &op)
{
    using G = Geo<FMT, MS>;
    const int row = c.wave * 64 + 32 * j + (c.lane & 31), g = c.lane >> 5;
#pragma unroll
    for (int h = 0; h < G::CCH / 2; ++h) {
        const int lc = g * (G::CCH / 2) + h;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(
            st + G::XBYTES + (row * G::CCH + (lc ^ cswz<FMT>(row))) * 16);
#pragma unroll
        for (int w = 0; w < 4; ++w)
            op.raw[j][4 * h + w] = v[w];
    }
    if constexpr (SWIDE) {
        if constexpr (U == 0) {
            // MXFP4: the second four steps of a group of eight take its other half
            if (G::SSTEPS == 2 && (t & 4)) {
                op.grp[j][0] = op.grp[j][2];
                op.grp[j][1] = op.grp[j][3];
            } else {
                op.grp[j] = *reinterpret_cast<const u32x4 *>(c.sring + row * 16);
            }
        }
    } else {
        op.grp[j][0] = *reinterpret_cast<const uint32_t *>(c.sring + t % 3 * G::SSTEP +
                                                           g * (BN * 4) + row * 4);
    }
}

template <int FMT, int MS, bool SWIDE, int U>
__device__ inline void scale_value(int lane, int j, Ops<FMT, MS> &op)
{
    // SWIDE: this lane half's part of the group's dword; otherwise the scale itself
    const int g = SWIDE ? lane >> 5 : 0;
    const uint32_t d = op.grp[j][SWIDE ? U / Geo<FMT, MS>::SSTEPS : 0];
    if constexpr (FMT == QL_FMT_MXFP4)
        op.sc[j] = mx_scale(d >> ((SWIDE ? 16 * (U & 1) : 0) + 8 * g) & 255u);
    else
        op.sc[j] = plane_scale((float)__builtin_bit_cast(_Float16, (uint16_t)(d >> (16 * g))));
}

// word w (two k) of fragment j, chunk q
template <int FMT, int MS>
__device__ inline void weight_word(const Ops<FMT, MS> &op, int j, int q, int w,
                                   u32x4 (&b)[NS][Geo<FMT, MS>::PLANES])
{
    // (pinned to where it is written: the words would otherwise gather behind the
    // chunk's last MFMA)
    uint32_t hi, lo;
    decode_word<FMT>(op.raw[j], 4 * q + w, op.sc[j], hi, lo);
    dma_pin(hi);
    b[j][0][w] = hi;
    if constexpr (Geo<FMT, MS>::PLANES == 2) {
        dma_pin(lo);
        b[j][1][w] = lo;
    }
}

// The MFMAs of chunk Q of step t (U = t % 4), and behind each, in a group that
// the compiler keeps together, a share of the next chunk's operands: of this
// stage (Q < 3) or with NEXT of the next one (nxt).
template <int FMT, int MS, bool SWIDE, int U, int Q, bool NEXT>
__device__ inline void chunk(const Ctx<FMT, MS, SWIDE> &c, const uint8_t *cur, const uint8_t *nxt,
                             int t, Ops<FMT, MS> &op, f32x16 (&acc)[MS][NS])
{
    constexpr int P = Geo<FMT, MS>::PLANES, KK = MS * NS * P, UN = (U + 1) & 3;
    constexpr int W0 = Q < 3 ? 0 : KK / 2, PER = (8 + KK - W0 - 1) / (KK - W0);  // words per MFMA
    static_assert(NS == 2, "8 words");
    u32x4 an[MS], bn[NS][P];
#pragma unroll
    for (int k = 0; k < KK; ++k) {
        const int v = P - 1 - k / (MS * NS), i = k / NS % MS, j = k % NS;
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, op.a[i]), __builtin_bit_cast(bf16x8, op.b[j][v]), acc[i][j],
            0, 0, 0);
        if constexpr (Q < 3 || NEXT) {
            if (Q == 3 && k < NS)
                read_weights<FMT, MS, SWIDE, UN>(c, nxt, t + 1, k, op);
            if (k < 2 * MS && k % 2 == 0)
                an[k / 2] = read_x(Q < 3 ? cur : nxt, c.lane, Q < 3 ? Q + 1 : 0, k / 2);
            if (Q == 3 && k == W0 - 1) {
#pragma unroll
                for (int jj = 0; jj < NS; ++jj)
                    scale_value<FMT, MS, SWIDE, UN>(c.lane, jj, op);
            }
            if (k >= W0) {
#pragma unroll
                for (int w = (k - W0) * PER; w < (k - W0 + 1) * PER; ++w)
                    if (w < 8)
                        weight_word<FMT, MS>(op, w / 4, Q < 3 ? Q + 1 : 0, w % 4, bn);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (Q < 3 || NEXT) {
#pragma unroll
        for (int i = 0; i < MS; ++i)
            op.a[i] = an[i];
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int v = 0; v < P; ++v)
                op.b[j][v] = bn[j][v];
    }
}

// Step t (U: its place in the loop's four).  TAIL: one of the last four, all
// conditions known, so that a step is one basic block.  Chunks 0-2 prepare their
// successors from the stage; then all of the stage is in registers, the next one
// has landed (loads land in order: what was issued after it may be in flight), and
// behind the barrier the stage's slot is refilled while chunk 3 runs and prepares
// the next stage's first one.
template <int FMT, int MS, bool SWIDE, int U, bool TAIL>
__device__ inline void step(Ctx<FMT, MS, SWIDE> &c, int t, int &slot, Ops<FMT, MS> &op,
                            f32x16 (&acc)[MS][NS])
{
    using G = Geo<FMT, MS>;
    constexpr int NST = G::NST;
    constexpr bool LAST = TAIL && U == 3;                   // t + 1 == ns
    constexpr bool ISSUE = !TAIL || U + NST < 4;            // t + NST < ns
    constexpr bool YOUNGER = NST == 3 && (!TAIL || U < 2);  // stage t + 2 is in flight
    const uint8_t *const cur = c.ring + slot * G::STAGE;
    const int nslot = slot + 1 == NST ? 0 : slot + 1;
    const uint8_t *const nxt = c.ring + nslot * G::STAGE;
    chunk<FMT, MS, SWIDE, U, 0, false>(c, cur, nxt, t, op, acc);
    chunk<FMT, MS, SWIDE, U, 1, false>(c, cur, nxt, t, op, acc);
    chunk<FMT, MS, SWIDE, U, 2, false>(c, cur, nxt, t, op, acc);
    if constexpr (!LAST) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        // a group of scales starts every 4 SSTEPS steps; the next one's are issued
        // behind its first step's barrier, before the stage
        const bool first = G::SSTEPS == 1 || !(t & 4);
        if constexpr (YOUNGER) {
            if (SWIDE && U == 1 && first)
                __builtin_amdgcn_s_waitcnt(dma_vmcnt(G::LOADS + 1));
            else
                __builtin_amdgcn_s_waitcnt(dma_vmcnt(G::LOADS + (SWIDE ? 0 : 2)));
        } else {
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(0));
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        if (SWIDE && U == 0 && first)
            issue_scales<FMT, MS, SWIDE>(c);
        if constexpr (ISSUE)
            issue<FMT, MS, SWIDE>(c, t + NST, slot);
        chunk<FMT, MS, SWIDE, U, 3, true>(c, cur, nxt, t, op, acc);
    } else {
        chunk<FMT, MS, SWIDE, U, 3, false>(c, cur, nxt, t, op, acc);
    }
    slot = nslot;
}

// SWIDE: scales 16 bytes at a time.  EPI: an epilogue beyond the output's type.
template <int FMT, int MS, bool GATED, bool SWIDE, bool EPI>
__global__ __launch_bounds__(THREADS, 2) void qgemm_tile_kernel(const TileArgs a)
{
    using G = Geo<FMT, MS>;
    constexpr int NST = G::NST, BM = G::BM, GROUP_M = 16 / MS;
    constexpr int COLS = GATED ? BN / 2 : BN;  // output columns of a tile
    __shared__ __align__(16) uint8_t ring[G::LDS];
    const int M = a.M, N = a.N, K = a.K, nb = K >> 5;
    const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + COLS - 1) / COLS;
    // each XCD takes a contiguous range of the tiles, in groups of 4 row tiles
    // walked row tile fastest
    const int p = (int)blockIdx.x, grid = (int)gridDim.x;
    const int gq = grid >> 3, gr = grid & 7, xcd = p & 7, idx = p >> 3;
    const int tile = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int gid = tile / (GROUP_M * tiles_n), within = tile - gid * (GROUP_M * tiles_n);
    const int gsz = min(tiles_m - gid * GROUP_M, GROUP_M);
    const int m0 = (gid * GROUP_M + within % gsz) * BM, n0 = within / gsz * COLS;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;

    // (an odd number of steps gets one of zeros)
    const int plane_steps = (nb + 1) >> 1, ns = (plane_steps * a.planes + 1) & ~1;

    Ctx<FMT, MS, SWIDE> c;
    c.ring = ring;
    c.sring = ring + NST * G::STAGE;
    c.wave = wave;
    c.lane = lane;
    c.plane_steps = plane_steps;
    c.planes = a.planes;
    c.nb = nb;
    c.ik = c.sk = 0;
    c.plane_skip = a.plane_bytes - (int64_t)plane_steps * 128;
    c.x = static_cast<const uint8_t *>(a.X) + (int64_t)m0 * K * 2;
    // per-lane offsets within the tile; rows past the end repeat the last one
#pragma unroll
    for (int r = 0; r < G::XLOADS; ++r) {
        const int i = r * THREADS + tid, row = i >> 3, lc = (i & 7) ^ xswz(row);
        c.xoff[r] = (uint32_t)((min(m0 + row, M - 1) - m0) * K * 2 + lc * 16);
    }
    const uint8_t *const cbase[2] = {a.codes[0], a.codes[GATED ? 1 : 0]};
    const uint8_t *const sbase[2] = {static_cast<const uint8_t *>(a.scales[0]),
                                     static_cast<const uint8_t *>(a.scales[GATED ? 1 : 0])};
    const int crow = nb * (G::CROW / 2), srow = nb * G::SB;
    // (a wavefront's chunks of one load lie in rows of one projection: 64 lanes
    // cover 32 rows of 2 chunks, or 16 of 4)
#pragma unroll
    for (int r = 0; r < G::CLOADS; ++r) {
        const int i = r * THREADS + tid, row = i / G::CCH, lc = (i % G::CCH) ^ cswz<FMT>(row);
        const int n = min(n0 + tile_row<GATED>(row), N - 1) - n0;
        const int up = GATED ? __builtin_amdgcn_readfirstlane((row >> 5) & 1) : 0;
        c.cptr[r] = cbase[up] + (int64_t)n0 * crow;
        c.coff[r] = (uint32_t)(n * crow + lc * 16);
    }
    // a wavefront's 64 scale rows: of a gated pair, half of each projection
    c.sp = sbase[GATED ? (tid >> 5) & 1 : 0] +
           (int64_t)min(n0 + tile_row<GATED>(tid), N - 1) * srow;

    f32x16 acc[MS][NS];
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.f;

    {
        if (SWIDE)
            issue_scales<FMT, MS, SWIDE>(c);
#pragma unroll
        for (int t = 0; t < NST; ++t)
            issue<FMT, MS, SWIDE>(c, t, t);
        // stage 0: the younger ones may be in flight (ns >= 4 > NST)
        __builtin_amdgcn_s_waitcnt(dma_vmcnt((NST - 1) * (G::LOADS + (SWIDE ? 0 : 2))));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        Ops<FMT, MS> op;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            read_weights<FMT, MS, SWIDE, 0>(c, c.ring, 0, j, op);
            scale_value<FMT, MS, SWIDE, 0>(lane, j, op);
        }
#pragma unroll
        for (int i = 0; i < MS; ++i)
            op.a[i] = read_x(c.ring, lane, 0, i);
#pragma unroll
        for (int w = 0; w < 8; ++w)
            weight_word<FMT, MS>(op, w / 4, 0, w % 4, op.b);
        int slot = 0, t = 0;
        if (!SWIDE && (ns & 2)) {  // (then ns is 6 at least: the tail follows)
            step<FMT, MS, SWIDE, 0, false>(c, 0, slot, op, acc);
            step<FMT, MS, SWIDE, 1, false>(c, 1, slot, op, acc);
            t = 2;
        }
#pragma unroll 1
        for (; t + 4 < ns; t += 4) {
            step<FMT, MS, SWIDE, 0, false>(c, t, slot, op, acc);
            step<FMT, MS, SWIDE, 1, false>(c, t + 1, slot, op, acc);
            step<FMT, MS, SWIDE, 2, false>(c, t + 2, slot, op, acc);
            step<FMT, MS, SWIDE, 3, false>(c, t + 3, slot, op, acc);
        }
        step<FMT, MS, SWIDE, 0, true>(c, t, slot, op, acc);
        step<FMT, MS, SWIDE, 1, true>(c, t + 1, slot, op, acc);
        step<FMT, MS, SWIDE, 2, true>(c, t + 2, slot, op, acc);
        step<FMT, MS, SWIDE, 3, true>(c, t + 3, slot, op, acc);
    }
    __syncthreads();  // the ring is free: the 32 x 32 tiles turn through patches of it

    float *const patch = reinterpret_cast<float *>(ring) + wave * STRIP_PATCH;
    if constexpr (GATED) {
        strip_gated(a.gate, M, N, m0, n0 + wave * 32, patch, lane, acc);
    } else {
        strip_store<EPI>(a.ep, a.Y, M, N, m0, n0 + wave * 64, patch, lane, acc,
                         epi_vec_ok(a.ep, a.Y, N), true);
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

static int64_t tile_tiles(int rows, int64_t M, int64_t N, bool gated)
{
    const int cols = gated ? BN / 2 : BN;
    return (M + rows - 1) / rows * ((N + cols - 1) / cols);
}

// scales in 16-byte chunks: whole groups in a row, 16-byte aligned
static bool scales_wide(int fmt, int64_t K, const void *scales0, const void *scales1)
{
    return K % (fmt == QL_FMT_MXFP4 ? 512 : 256) == 0 &&
           (((uintptr_t)scales0 | (uintptr_t)scales1) & 15) == 0;
}

// (four steps at least: the loop's last round)
bool tile_takes(int64_t K) { return K >= 224 && K < ((int64_t)1 << 22); }

// us of tiles of 128 and 64 rows: fixed; of a 64-k step where a tile has its CU to
// itself (latency, and rising with the share of the CUs that work), and per tile of a
// CU that several share.  Products with MXFP4 weights, gated pairs of MXFP4, of q4 and
// int8 (twice the matrix instructions), and of these where scales come one by one (whose
// 128-row tiles do not fit the registers).  Measured, 64 / 128 rows: product 6144 x
// 1536 at 512 rows 14.6 / 21.2, at 768 22.3 / 21.8, 1536 x 6144 at 2048 46.0 / 67.9,
// fp32 at 1536 140 / 206; pairs 6144 x 1536 at 256 rows 17.1 / 25.8, at 2048 78.5 / 70.9,
// q4 at 256 rows 32.5 / 44.6, at 512 54.4 / 47.4; scales one by one, int8 2048 x 1056 at
// 1748 rows 46.6 / 65.6, q4 4096 x 1504 at 1100 91.4 / 104, at 2048 122 / 109.
struct TileRate {
    double fixed, alone, rise, shared;
};
constexpr TileRate TILE_RATES[4][2] = {{{5.2, 0.63, 0.08, 0.88}, {4.5, 0.38, 0.06, 0.49}},
                                       {{10.0, 0.62, 0.16, 0.86}, {7.0, 0.36, 0.09, 0.50}},
                                       {{10.0, 1.42, 0.30, 1.82}, {7.0, 0.96, 0.10, 1.14}},
                                       {{10.0, 2.30, 0.40, 2.20}, {7.0, 1.05, 0.15, 1.25}}};

double tile_us(int fmt, bool xf32, bool gated, int64_t M, int64_t N, int64_t K, int cus, int *rows)
{
    const double steps = (double)((K + 63) / 64) * (xf32 ? 3 : 1);
    const int kind = !gated ? 0 : fmt == QL_FMT_MXFP4 ? 1 : K % 256 == 0 ? 2 : 3;
    double best = 1e30;
    for (int h = 0; h < 2; ++h) {
        const TileRate &t = TILE_RATES[kind][h];
        const int tile = h ? 64 : 128;
        const int64_t tiles = tile_tiles(tile, M, N, gated);
        if (tiles > MAX_WORKGROUPS)
            continue;
        const double r = (double)tiles / cus, up = std::ceil(r);
        const double us = t.fixed + steps * (r <= 1.0 ? t.alone + t.rise * r
                                                      : t.shared * (r + 0.4 * (up - r)));
        if (us < best) {
            best = us;
            *rows = tile;
        }
    }
    return best + (xf32 ? 2.0 + 10.0 * (double)M * (double)K / 5e6 : 0.0);
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
    const dim3 grid((unsigned)tile_tiles(a.rows, a.M, a.N, gated)), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    const bool swide = scales_wide(fmt, a.K, a.scales[0], a.scales[1]);
    auto with = [&](auto fmtc, auto gatedc, auto epic) {
        constexpr int F = decltype(fmtc)::value;
        constexpr bool GD = decltype(gatedc)::value, E = decltype(epic)::value;
        if (a.rows == 64)
            swide ? go(qgemm_tile_kernel<F, 2, GD, true, E>)
                  : go(qgemm_tile_kernel<F, 2, GD, false, E>);
        else
            swide ? go(qgemm_tile_kernel<F, 4, GD, true, E>)
                  : go(qgemm_tile_kernel<F, 4, GD, false, E>);
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
