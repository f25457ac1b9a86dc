// bf16 products of the gated feed-forward's backward pass, fp32 accumulation:
//
//   C[r][s] = sum over the segments of  sum_c A(r, c) B(c, s)
//
//   dX  (TRA = false): A = dG [M][N] then dU, rows along the reduction;
//                      B = the dequantized gate weights [N][K], then the up's
//                      (q4, int8: each as the sum of two bf16, four segments)
//   dW  (TRA = true):  A = dG or dU [M][N], the reduction over its rows;
//                      B = X [M][K] (one problem per projection)
//
// Matrix instruction v_mfma_f32_32x32x16_bf16: lane l holds A[l % 32][8 (l /
// 32) + e] and B[8 (l / 32) + e][l % 32].  An operand stored with the
// reduction along its rows is read from LDS with the transposing read
// (ds_read_b64_tr_b16: 16 lanes that address 4 rows x 4 runs of 4 columns
// receive 4 rows of one column each), so neither needs a transposed copy.
//
// Tile: 4 wavefronts compute 128 x 256, each a strip of 64 columns (4 x 2 MFMA
// tiles), or 64 x 256 where tiles are few (twice the wavefronts).  Direct-to-LDS loads
// fill a ring of stages of 32 c: three (64 rows: four; two workgroups per CU), or six
// where there is no more than a workgroup for each CU.
// The barrier of a stage sits before its last 16-c chunk; behind every MFMA goes a
// share of the next chunk's LDS reads.  Chunks of 16 bytes are XOR-swizzled
// against bank conflicts.  Reductions that do not divide into whole stages end in
// one filled up from a page of zeros.
//
// Few tiles: the reduction is cut into parts whose fp32 sums another launch
// adds in order (split_sum_kernel).
//
// Bound: the issue of matrix instructions.  While a CU holds a workgroup its matrix cores
// are busy 0.56 (dX) and 0.51 (dW) of the cycles, its LDS 0.24; wavefronts wait 0.45 of
// theirs for an instruction's unit, 0.22 for data or a barrier.  Then the clock (1.75 GHz of
// 2.4 in a run of 32768 rows, where the cores are busy 0.61 to 0.64) and the tail.  2048
// rows, N = 4096, K = 1536 (51.5 Gflop each): dX 53.5 us in 5 parts (480 workgroups) and
// 14.7 us for their sum, dW 59.6 us (384 workgroups on 512 places, a quarter of them idle).
#include <algorithm>

#include "dma.h"
#include "internal.h"
#include "mx.h"
#include "strip.h"

namespace qlk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int BN = 256, BC = 32;
constexpr int NS = 2;  // MFMA tiles of a wavefront across
constexpr int BBYTES = BN * BC * 2, BLOADS = BBYTES / 16 / THREADS;

// MS: blocks of 32 rows of the tile.
template <int MS>
struct Geo {
    static constexpr int BM = 32 * MS, ABYTES = BM * BC * 2, STAGE = ABYTES + BBYTES;
    static constexpr int ALOADS = ABYTES / 16 / THREADS, LOADS = ALOADS + BLOADS;
};

__device__ __align__(16) const uint32_t zeros[4] = {0, 0, 0, 0};

// swizzles of 16-byte chunks: rows of 4 chunks (reduction along the row; a cycle
// of a 16-byte read serves rows 0-3, 12-15, 20-27, or the others of 32), and rows
// of 8, 16 or 32 (reduction over rows)
__device__ inline int swz4(int row) { return ((row >> 2) & 3) ^ ((row >> 4) & 1) * 3; }
template <int LINES>
__device__ inline int swzt(int row)
{
    return (row & 3) << (LINES == 64 ? 1 : 2);
}

// Where the chunk in slot i of an operand's stage comes from: its byte offset
// in the matrix, from the tile's corner at (first line, first reduction index).
// LINES: BM or BN.  Lines past the end repeat the last one (`lines` are there);
// c: the chunk's first reduction index within the stage.
template <bool TR, int LINES>
__device__ inline uint32_t chunk_at(int i, int lines, int64_t ld, int &c)
{
    if constexpr (TR) {
        constexpr int CH = LINES / 8;
        const int row = i / CH, lc = (i % CH) ^ swzt<LINES>(row);
        c = row;
        return (uint32_t)((row * ld + min(lc * 8, lines - 8)) * 2);
    } else {
        const int row = i >> 2, lc = (i & 3) ^ swz4(row);
        c = lc * 8;
        return (uint32_t)((min(row, lines - 1) * ld + lc * 8) * 2);
    }
}

// fragment of 16-c chunk q: line `line` + lane % 32, c = 16 q + 8 (lane / 32) + e
template <bool TR, int LINES>
__device__ inline bf16x8 fragment(const uint8_t *st, int line, int q, int lane)
{
    const int g = lane >> 5;
    if constexpr (TR) {
        const int row = 16 * q + 8 * g + ((lane & 15) >> 2);
        const int unit = line / 4 + 4 * ((lane >> 4) & 1) + (lane & 3);  // of 4 lines, 8 bytes
        auto at = [&](int r) {
            return st + r * (LINES * 2) + ((unit >> 1) ^ swzt<LINES>(r)) * 16 + (unit & 1) * 8;
        };
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)at(row));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)at(row + 4));
        const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
        return __builtin_bit_cast(bf16x8, u32x4{l[0], l[1], h[0], h[1]});
    } else {
        const int row = line + (lane & 31), lc = 2 * q + g;
        return __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const u32x4 *>(st + (row * 4 + (lc ^ swz4(row))) * 16));
    }
}

// What a lane needs of a tile, fixed for the whole reduction, and how far the
// loads have come.
template <int MS>
struct Ctx {
    uint8_t *ring;
    uint32_t aoff[Geo<MS>::ALOADS], boff[BLOADS];
    int ac[Geo<MS>::ALOADS], bc[BLOADS];  // each chunk's first reduction index in its stage
    const uint8_t *A, *B;        // of the next stage
    int64_t astep, bstep;        // from one stage to the next
    int seg, c0;                 // of the next stage
    int wave, lane;
};

template <bool TRA, int MS>
__device__ inline void start_segment(const GemmArgs &a, Ctx<MS> &c, int prob, int m0, int n0)
{
    const bool many = a.segs > 1;
    c.A = reinterpret_cast<const uint8_t *>(a.A[many ? c.seg : prob] +
                                            (TRA ? c.c0 * a.lda + m0 : m0 * a.lda + c.c0));
    c.B = reinterpret_cast<const uint8_t *>(a.B[many ? c.seg : 0] + c.c0 * a.ldb + n0);
}

template <bool TRA, int MS>
__device__ inline void issue(const GemmArgs &a, Ctx<MS> &c, int prob, int m0, int n0, int slot)
{
    constexpr int ALOADS = Geo<MS>::ALOADS, ABYTES = Geo<MS>::ABYTES, STAGE = Geo<MS>::STAGE;
    const uint32_t base = dma_lds(c.ring + slot * STAGE) + c.wave * 1024;
    if (c.c0 + BC <= a.C) {
#pragma unroll
        for (int i = 0; i < ALOADS; ++i)
            dma_load16(c.A, c.aoff[i], base + i * THREADS * 16);
#pragma unroll
        for (int i = 0; i < BLOADS; ++i)
            dma_load16(c.B, c.boff[i], base + ABYTES + i * THREADS * 16);
    } else {
#pragma unroll
        for (int i = 0; i < ALOADS; ++i)
            dma_load16_at(c.c0 + c.ac[i] < a.C ? c.A + c.aoff[i] : (const uint8_t *)zeros,
                          base + i * THREADS * 16);
#pragma unroll
        for (int i = 0; i < BLOADS; ++i)
            dma_load16_at(c.c0 + c.bc[i] < a.C ? c.B + c.boff[i] : (const uint8_t *)zeros,
                          base + ABYTES + i * THREADS * 16);
    }
    c.c0 += BC;
    c.A += c.astep;
    c.B += c.bstep;
    if (c.c0 >= a.C && c.seg + 1 < a.segs) {
        ++c.seg;
        c.c0 = 0;
        start_segment<TRA, MS>(a, c, prob, m0, n0);
    }
}

// The MFMAs of a 16-c chunk, and behind each, in a group that the compiler keeps
// together, a share of the operands of chunk QN of stage nxt.
template <bool TRA, int MS, int QN>
__device__ inline void chunk(const Ctx<MS> &c, const uint8_t *nxt, bf16x8 (&av)[MS], bf16x8 (&bv)[NS],
                             f32x16 (&acc)[MS][NS])
{
    constexpr int BM = Geo<MS>::BM, ABYTES = Geo<MS>::ABYTES;
    bf16x8 an[MS], bn[NS];
#pragma unroll
    for (int k = 0; k < MS * NS; ++k) {
        const int i = k / NS, j = k % NS;
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[i], bv[j], acc[i][j], 0, 0, 0);
        // (two fragments at a time: they have to be there by the chunk's end)
        if (k == 0) {
#pragma unroll
            for (int jj = 0; jj < NS; ++jj)
                bn[jj] = fragment<true, BN>(nxt + ABYTES, c.wave * 64 + 32 * jj, QN, c.lane);
        } else if (k <= MS / 2) {
            an[2 * k - 2] = fragment<TRA, BM>(nxt, 32 * (2 * k - 2), QN, c.lane);
            an[2 * k - 1] = fragment<TRA, BM>(nxt, 32 * (2 * k - 1), QN, c.lane);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < MS; ++i)
        av[i] = an[i];
#pragma unroll
    for (int j = 0; j < NS; ++j)
        bv[j] = bn[j];
}

template <bool TRA, int MS, int NST>
__global__ __launch_bounds__(THREADS, NST > 4 ? 1 : 2) void gemm_bf16_kernel(const GemmArgs a)
{
    using G = Geo<MS>;
    constexpr int BM = G::BM, ALOADS = G::ALOADS, LOADS = G::LOADS, ABYTES = G::ABYTES;
    constexpr int STAGE = G::STAGE, GROUP_M = 16 / MS;
    __shared__ __align__(16) uint8_t ring[NST * STAGE];
    const int tiles_m = (a.R + BM - 1) / BM, tiles_n = (a.S + BN - 1) / BN;
    // each XCD takes a contiguous range of the tiles, in groups of 4 row tiles
    // walked row tile fastest, all tiles of a part before the next one's: tiles of one
    // part share operands (q4 at 2048 rows, dX of 2752 x 1024 70 -> 67 us)
    const int p = (int)blockIdx.x, grid = (int)gridDim.x;
    const int gq = grid >> 3, gr = grid & 7, xcd = p & 7, idx = p >> 3;
    const int local = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int all_tiles = grid / a.parts;  // of all problems
    const int part = local / all_tiles, pt = local - part * all_tiles;
    const int prob = pt / (tiles_m * tiles_n), tile = pt - prob * (tiles_m * tiles_n);
    const int gid = tile / (GROUP_M * tiles_n), within = tile - gid * (GROUP_M * tiles_n);
    const int gsz = min(tiles_m - gid * GROUP_M, GROUP_M);
    const int m0 = (gid * GROUP_M + within % gsz) * BM, n0 = within / gsz * BN;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;

    // the reduction: `segs` segments of C each, in whole stages of BC
    const int seg_steps = (a.C + BC - 1) / BC, all_steps = seg_steps * a.segs;
    const int per = (all_steps + a.parts - 1) / a.parts;
    const int s0 = part * per, ns = min(all_steps, s0 + per) - s0;

    f32x16 acc[MS][NS];
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.f;

    if (ns > 0) {
        Ctx<MS> c;
        c.ring = ring;
        c.wave = wave;
        c.lane = lane;
#pragma unroll
        for (int i = 0; i < ALOADS; ++i)
            c.aoff[i] = chunk_at<TRA, BM>(i * THREADS + tid, a.R - m0, a.lda, c.ac[i]);
#pragma unroll
        for (int i = 0; i < BLOADS; ++i)
            c.boff[i] = chunk_at<true, BN>(i * THREADS + tid, a.S - n0, a.ldb, c.bc[i]);
        c.astep = (TRA ? BC * a.lda : BC) * 2;
        c.bstep = BC * a.ldb * 2;
        c.seg = s0 / seg_steps;
        c.c0 = (s0 - c.seg * seg_steps) * BC;
        start_segment<TRA, MS>(a, c, prob, m0, n0);
#pragma unroll 1
        for (int t = 0; t < NST && t < ns; ++t)
            issue<TRA, MS>(a, c, prob, m0, n0, t);
        dma_wait<LOADS, NST - 1>(min(ns, NST) - 1);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        bf16x8 av[MS], bv[NS];
#pragma unroll
        for (int j = 0; j < NS; ++j)
            bv[j] = fragment<true, BN>(ring + ABYTES, wave * 64 + 32 * j, 0, lane);
#pragma unroll
        for (int i = 0; i < MS; ++i)
            av[i] = fragment<TRA, BM>(ring, 32 * i, 0, lane);
        int slot = 0;
        for (int t = 0; t < ns; ++t) {
            uint8_t *const cur = ring + slot * STAGE;
            const int nslot = slot + 1 == NST ? 0 : slot + 1;
            chunk<TRA, MS, 1>(c, cur, av, bv, acc);
            // all of the stage is in registers; the next one has landed where only
            // those younger than it are in flight (loads land in order); behind the
            // barrier the stage's slot is refilled while its last chunk runs and
            // prepares the next stage's first (after the last stage: from whatever
            // the next slot holds, never multiplied)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (t + NST < ns)
                __builtin_amdgcn_s_waitcnt(dma_vmcnt((NST - 2) * LOADS));
            else
                dma_wait<LOADS, NST - 2>(min(ns - 2 - t, NST - 2));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (t + NST < ns)
                issue<TRA, MS>(a, c, prob, m0, n0, slot);
            chunk<TRA, MS, 0>(c, ring + nslot * STAGE, av, bv, acc);
            slot = nslot;
        }
    }
    __syncthreads();  // the ring is free: the 32 x 32 tiles turn through patches of it

    const bool to_part = a.parts > 1;
    const int64_t RS = (int64_t)a.R * a.S;
    Epilogue e{};
    e.ybf16 = !to_part && a.outbf16;
    float *const Y = to_part ? a.part + ((int64_t)prob * a.parts + part) * RS
                             : static_cast<float *>(a.out[prob]);
    // (S % 8 == 0 and aligned outputs: whole groups of four)
    strip_store<false>(e, Y, a.R, a.S, m0, n0 + wave * 64,
                       reinterpret_cast<float *>(ring) + wave * STRIP_PATCH, lane, acc, true,
                       !to_part);
}

// Column sums of bf16 matrices [M][N] (bias gradients), in a fixed order: a
// workgroup owns 64 columns of one, its threads rows t / 8, t / 8 + 32, ... of 8
// columns each, added up in LDS.  Bound: the latency of M / 32 dependent rows a thread, on
// half of the CUs: 2048 x 4096 of both 23 us (33.6 MB, 6.6 us of a copy).
__global__ __launch_bounds__(256) void column_sums_kernel(const uint16_t *dG, const uint16_t *dU,
                                                          float *dbg, float *dbu, int M, int N)
{
    __shared__ float red[32][65];
    const uint16_t *const D = blockIdx.y ? dU : dG;
    float *const out = blockIdx.y ? dbu : dbg;
    const int c0 = (int)blockIdx.x * 64, cg = threadIdx.x & 7, rg = threadIdx.x >> 3;
    const int col = c0 + 8 * cg;
    float s[8] = {};
    if (out && col < N)
        for (int64_t m = rg; m < M; m += 32) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(D + m * N + col);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[2 * e] += __uint_as_float(w[e] << 16);
                s[2 * e + 1] += __uint_as_float(w[e] & 0xFFFF0000u);
            }
        }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        red[rg][8 * cg + e] = s[e];
    __syncthreads();
    if (threadIdx.x < 64 && out && c0 + (int)threadIdx.x < N) {
        float t = 0.f;
        for (int r = 0; r < 32; ++r)
            t += red[r][threadIdx.x];
        out[c0 + threadIdx.x] = t;
    }
}

}  // namespace

int64_t gemm_tiles(int rows, int64_t R, int64_t S)
{
    return (R + rows - 1) / rows * ((S + BN - 1) / BN);
}

int gemm_parts(int64_t tiles, int64_t R, int64_t S, int64_t C, GemmCost cost, int cus,
               double *best_us)
{
    // a part more costs a sum's round trip through memory at 5 TB/s, and the first
    // one the sum's launch
    const int64_t steps = (C + BC - 1) / BC;
    int best = 1;
    double us = 0.0;  // (of the best so far)
    for (int p = 1; p <= 32 && p * 8 <= std::max<int64_t>(8, steps); ++p) {
        const int64_t rounds = (tiles * p + cus - 1) / cus;
        const double stage = rounds == 1 ? cost.alone_us : rounds * cost.shared_us;
        const double t = (double)((steps + p - 1) / p) * stage + 3.0 * rounds +
                         (p > 1 ? 4.0 + 8.0 * p * (double)(R * S) / 5e6 : 0.0);
        if (p == 1 || t < us) {
            best = p;
            us = t;
        }
    }
    if (best_us)
        *best_us = us;
    return best;
}

hipError_t launch_gemm_bf16(bool tra, const GemmArgs &a, int problems, hipStream_t stream)
{
    const int64_t wgs = gemm_tiles(a.rows, a.R, a.S) * problems * a.parts;
    const dim3 grid((unsigned)wgs), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    const bool alone = wgs <= current_cus();
    auto with = [&](auto trac) {
        constexpr bool T = decltype(trac)::value;
        if (a.rows == 64)
            alone ? go(gemm_bf16_kernel<T, 2, 6>) : go(gemm_bf16_kernel<T, 2, 4>);
        else
            alone ? go(gemm_bf16_kernel<T, 4, 6>) : go(gemm_bf16_kernel<T, 4, 3>);
    };
    tra ? with(std::true_type{}) : with(std::false_type{});
    return hipGetLastError();
}

hipError_t launch_column_sums(const uint16_t *dG, const uint16_t *dU, float *dbg, float *dbu, int M,
                              int N, hipStream_t stream)
{
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((N + 63) / 64), 2), dim3(256), 0, stream,
                       dG, dU, dbg, dbu, M, N);
    return hipGetLastError();
}

}  // namespace qlk
