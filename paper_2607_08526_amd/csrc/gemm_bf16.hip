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
// tiles).  Direct-to-LDS loads fill a ring of three stages of 32 c (72 KB, two
// workgroups per CU); one barrier per stage: at it a wavefront's stage has
// landed and the slot of the one before is free for the next but one.  Chunks of
// 16 bytes are XOR-swizzled against bank conflicts.  Reductions that do not
// divide into whole stages end in one filled up from a page of zeros.
//
// Few tiles: the reduction is cut into parts whose fp32 sums another launch
// adds in order (split_sum_kernel).
#include <algorithm>

#include "dma.h"
#include "internal.h"
#include "mx.h"

namespace qlk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int BM = 128, BN = 256, BC = 32, NST = 3;
constexpr int MS = 4, NS = 2;  // MFMA tiles of a wavefront
constexpr int ABYTES = BM * BC * 2, BBYTES = BN * BC * 2, STAGE = ABYTES + BBYTES;
constexpr int ALOADS = ABYTES / 16 / THREADS, BLOADS = BBYTES / 16 / THREADS;
constexpr int LOADS = ALOADS + BLOADS;
constexpr int GROUP_M = 4;

__device__ __align__(16) const uint32_t zeros[4] = {0, 0, 0, 0};

// swizzles of 16-byte chunks: rows of 4 chunks (reduction along the row; a cycle
// of a 16-byte read serves rows 0-3, 12-15, 20-27, or the others of 32), and rows
// of 16 or 32 (reduction over rows)
__device__ inline int swz4(int row) { return ((row >> 2) & 3) ^ ((row >> 4) & 1) * 3; }
__device__ inline int swzt(int row) { return (row & 3) << 2; }

// Where the chunk in slot i of an operand's stage comes from: its byte offset
// in the matrix, from the tile's corner at (first line, first reduction index).
// LINES: BM or BN.  Lines past the end repeat the last one (`lines` are there);
// c: the chunk's first reduction index within the stage.
template <bool TR, int LINES>
__device__ inline uint32_t chunk_at(int i, int lines, int64_t ld, int &c)
{
    if constexpr (TR) {
        constexpr int CH = LINES / 8;
        const int row = i / CH, lc = (i % CH) ^ swzt(row);
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
            return st + r * (LINES * 2) + ((unit >> 1) ^ swzt(r)) * 16 + (unit & 1) * 8;
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

template <bool TRA>
__global__ __launch_bounds__(THREADS, 2) void gemm_bf16_kernel(const GemmArgs a)
{
    __shared__ __align__(16) uint8_t ring[NST * STAGE];
    const int tiles_m = (a.R + BM - 1) / BM, tiles_n = (a.S + BN - 1) / BN;
    // each XCD takes a contiguous range of the tiles, in groups of 4 row tiles
    // walked row tile fastest; the parts of a tile are adjacent
    const int p = (int)blockIdx.x, G = (int)gridDim.x;
    const int gq = G >> 3, gr = G & 7, xcd = p & 7, idx = p >> 3;
    const int local = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int part = local % a.parts, pt = local / a.parts;
    const int prob = pt / (tiles_m * tiles_n), tile = pt - prob * (tiles_m * tiles_n);
    const int gid = tile / (GROUP_M * tiles_n), within = tile - gid * (GROUP_M * tiles_n);
    const int gsz = min(tiles_m - gid * GROUP_M, GROUP_M);
    const int m0 = (gid * GROUP_M + within % gsz) * BM, n0 = within / gsz * BN;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, g = lane >> 5;

    // the reduction: `segs` segments of C each, in whole stages of BC
    const int seg_steps = (a.C + BC - 1) / BC, all_steps = seg_steps * a.segs;
    const int per = (all_steps + a.parts - 1) / a.parts;
    const int s0 = part * per, s1 = min(all_steps, s0 + per);

    uint32_t aoff[ALOADS], boff[BLOADS];
    int ac[ALOADS], bc[BLOADS];
#pragma unroll
    for (int i = 0; i < ALOADS; ++i)
        aoff[i] = chunk_at<TRA, BM>(i * THREADS + tid, a.R - m0, a.lda, ac[i]);
#pragma unroll
    for (int i = 0; i < BLOADS; ++i)
        boff[i] = chunk_at<true, BN>(i * THREADS + tid, a.S - n0, a.ldb, bc[i]);

    auto issue = [&](int s) {
        uint8_t *const st = ring + (s - s0) % NST * STAGE;
        const int seg = s / seg_steps;
        const int c0 = (s - seg * seg_steps) * BC;
        const int w = a.segs > 1 ? seg : prob;
        const uint8_t *const A = reinterpret_cast<const uint8_t *>(
            a.A[w] + (TRA ? c0 * a.lda + m0 : m0 * a.lda + c0));
        const uint8_t *const B =
            reinterpret_cast<const uint8_t *>(a.B[a.segs > 1 ? seg : 0] + c0 * a.ldb + n0);
        const uint32_t base = dma_lds(st);
        if (c0 + BC <= a.C) {
#pragma unroll
            for (int i = 0; i < ALOADS; ++i)
                dma_load16(A, aoff[i], base + (i * THREADS + wave * 64) * 16);
#pragma unroll
            for (int i = 0; i < BLOADS; ++i)
                dma_load16(B, boff[i], base + ABYTES + (i * THREADS + wave * 64) * 16);
        } else {
#pragma unroll
            for (int i = 0; i < ALOADS; ++i)
                dma_load16_at(c0 + ac[i] < a.C ? A + aoff[i] : (const uint8_t *)zeros,
                              base + (i * THREADS + wave * 64) * 16);
#pragma unroll
            for (int i = 0; i < BLOADS; ++i)
                dma_load16_at(c0 + bc[i] < a.C ? B + boff[i] : (const uint8_t *)zeros,
                              base + ABYTES + (i * THREADS + wave * 64) * 16);
        }
    };

    f32x16 acc[MS][NS];
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.f;

    if (s0 < s1)
        issue(s0);
    if (s0 + 1 < s1)
        issue(s0 + 1);
    for (int s = s0; s < s1; ++s) {
        // loads land in order: all but the next stage's
        if (s + 1 < s1)
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(LOADS));
        else
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(0));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        if (s + 2 < s1)
            issue(s + 2);
        const uint8_t *const st = ring + (s - s0) % NST * STAGE;
#pragma unroll
        for (int q = 0; q < BC / 16; ++q) {
            bf16x8 av[MS], bv[NS];
#pragma unroll
            for (int j = 0; j < NS; ++j)
                bv[j] = fragment<true, BN>(st + ABYTES, wave * 64 + 32 * j, q, lane);
#pragma unroll
            for (int i = 0; i < MS; ++i)
                av[i] = fragment<TRA, BM>(st, 32 * i, q, lane);
#pragma unroll
            for (int i = 0; i < MS; ++i)
#pragma unroll
                for (int j = 0; j < NS; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[i], bv[j], acc[i][j],
                                                                        0, 0, 0);
        }
    }
    __syncthreads();  // the ring is free: every 32 x 32 tile turns through a patch of it

    float *const patch = reinterpret_cast<float *>(ring) + wave * 1024;
    const bool to_part = a.parts > 1;
    const int64_t RS = (int64_t)a.R * a.S;
    float *const F = to_part ? a.part + ((int64_t)prob * a.parts + part) * RS
                             : static_cast<float *>(a.out[prob]);
    const bool bf = !to_part && a.outbf16;
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                patch[(8 * (r >> 2) + 4 * g + (r & 3)) * 32 + l32] = acc[i][j][r];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = m0 + 32 * i + 8 * t + (lane >> 3);
                const int col = n0 + wave * 64 + 32 * j + 4 * (lane & 7);
                const f32x4 v = *reinterpret_cast<const f32x4 *>(patch + (8 * t + (lane >> 3)) * 32 +
                                                                 4 * (lane & 7));
                if (row >= a.R || col >= a.S)  // (S % 8 == 0: groups of four are whole)
                    continue;
                const int64_t at = (int64_t)row * a.S + col;
                if (bf)
                    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.out[prob]) + at) =
                        u32x2{mx_pack_bf16(v[0], v[1]), mx_pack_bf16(v[2], v[3])};
                else
                    *reinterpret_cast<f32x4 *>(F + at) = v;
            }
        }
}

// Column sums of bf16 matrices [M][N] (bias gradients), in a fixed order: a
// workgroup owns 64 columns of one, its threads rows t / 8, t / 8 + 32, ... of 8
// columns each, added up in LDS.
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

int64_t gemm_tiles(int64_t R, int64_t S) { return (R + BM - 1) / BM * ((S + BN - 1) / BN); }

int gemm_parts(int64_t tiles, int64_t C, int cus)
{
    // parts of at least 16 stages that fill the CUs about once
    const int64_t steps = (C + BC - 1) / BC;
    return (int)std::max<int64_t>(1, std::min<int64_t>(cus / std::max<int64_t>(1, tiles),
                                                       std::min<int64_t>(16, steps / 16)));
}

hipError_t launch_gemm_bf16(bool tra, const GemmArgs &a, int problems, hipStream_t stream)
{
    const dim3 grid((unsigned)(gemm_tiles(a.R, a.S) * problems * a.parts)), block(THREADS);
    if (tra)
        hipLaunchKernelGGL(gemm_bf16_kernel<true>, grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL(gemm_bf16_kernel<false>, grid, block, 0, stream, a);
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
