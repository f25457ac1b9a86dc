// The gradient of a gated pair's input, from the gradients of both projections
// and the compressed weights:
//
//   dX[m][k] = sum_n dG[m][n] Wg[n][k] + dU[m][n] Wu[n][k],   W = c * s
//
// The reduction runs over weight rows, so a matrix operand's 8 consecutive
// reduction indices lie in 8 rows: weights are converted to bf16 (MXFP4 exactly;
// q4 / int8 as the sum of two bf16, mx.h) into an LDS tile as they
// are stored, [32 n][256 k], and read with the transposing LDS read
// (ds_read_b64_tr_b16: 16 lanes that address 4 rows x 4 runs of 4 columns receive 4
// rows of one column each).  Matrix instruction v_mfma_f32_32x32x16_bf16 as in
// gemm_bf16.hip.
//
// Tile: 4 wavefronts compute 128 x 256, or 64 x 256 where tiles are few, each a strip of
// 64 columns.  A stage is 32 weight rows: dG's 128 x 32 and the codes move directly to LDS (as do scale
// dwords), and each thread converts one scale block of 32 codes, which it loaded
// itself, a share behind every MFMA of a stage's first 16-n chunk, into the other
// of two weight tiles; the barrier before the second chunk hands it over.  As codes
// the weights are 4 KB of a stage's 12 instead of 16 of 24: what bounds these
// products is the traffic into LDS (about 42 KB per us and CU).  MXFP4 two workgroups
// per CU, q4 and int8 one, with as many stages in flight as LDS holds.
//
// Few tiles: the reduction is cut into parts whose fp32 sums another launch
// adds in order (split_sum_kernel).
//
// Bound: the latency of a stage (0.45 to 1.0 us by format and tile, a quarter of it on
// the matrix cores) while a CU has one workgroup, and the sum's launch: q4, 107 rows, N
// = 2752, K = 1024 (1.2 Gflop): 23.6 us with the sum's 4.6.
#include <algorithm>

#include "dma.h"
#include "internal.h"
#include "mx.h"
#include "strip.h"

namespace qlk {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int BN = 256, BC = 32;
constexpr int NS = 2;  // MFMA tiles of a wavefront across

template <int FMT>
constexpr int WGS = FMT == QL_FMT_MXFP4 ? 2 : 1;  // workgroups per CU

// MS: blocks of 32 rows of the tile.
template <int FMT, int MS>
struct Geo {
    static constexpr int BM = 32 * MS;
    static constexpr int PLANES = FMT == QL_FMT_MXFP4 ? 1 : 2;
    static constexpr int CODES = FMT == QL_FMT_INT8 ? 32 : 16;  // bytes of a block's codes
    static constexpr int ABYTES = BM * BC * 2, CBYTES = THREADS * CODES, SBYTES = THREADS * 4;
    static constexpr int STAGE = ABYTES + CBYTES + SBYTES;
    static constexpr int BTILE = BC * BN * 2;  // a plane of a converted stage
    static constexpr int NST = (160 * 1024 / WGS<FMT> - 2 * PLANES * BTILE) / STAGE;
    static constexpr int LDS = NST * STAGE + 2 * PLANES * BTILE;
    static constexpr int ALOADS = ABYTES / 16 / THREADS, CLOADS = CODES / 16;
    static constexpr int LOADS = ALOADS + CLOADS + 1;
    static_assert(NS == 2, "two B fragments at a time");
    static_assert(NST >= 3 && (NST - 1) * LOADS < 63, "stages in flight");
};

__device__ __align__(16) const uint32_t zeros[4] = {0, 0, 0, 0};

// A: rows of 4 chunks of 16 bytes (a cycle of a 16-byte read serves rows 0-3,
// 12-15, 20-27, or the others of 32)
__device__ inline int aswz(int row) { return ((row >> 2) & 3) ^ ((row >> 4) & 1) * 3; }
// weight tile: rows of 32 chunks.  Reads take 64 bytes of each of 4 rows: the row
// picks the 64-byte piece; writes take chunk w of 8 blocks of two rows: row and
// block pick the chunk within it.
__device__ inline int bswz(int row, int chunk)
{
    return ((row & 3) << 2) ^ (((chunk >> 4) & 1) | (row & 1) << 1);
}

// A fragment of row block i: rows 32 i + lane % 32, n = 16 q + 8 (lane / 32) + e.
// at: a_at(lane, q) (the swizzle does not see i)
__device__ inline uint32_t a_at(int lane, int q)
{
    const int row = lane & 31;
    return (uint32_t)((row * 4 + ((2 * q + (lane >> 5)) ^ aswz(row))) * 16);
}
__device__ inline bf16x8 read_a(const uint8_t *st, uint32_t at, int i)
{
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(st + at + i * (32 * 64)));
}

// B fragment: columns line + lane % 32, the same n.  at: b_at(lane, line) (the
// swizzle does not see q: rows 8 apart look alike)
__device__ inline uint32_t b_at(int lane, int line)
{
    const int row = 8 * (lane >> 5) + ((lane & 15) >> 2);
    const int unit = line / 4 + 4 * ((lane >> 4) & 1) + (lane & 3);  // of 4 columns, 8 bytes
    return (uint32_t)(row * (BN * 2) + ((unit >> 1) ^ bswz(row, unit >> 1)) * 16 + (unit & 1) * 8);
}
__device__ inline bf16x8 read_b(const uint8_t *tile, uint32_t at, int q)
{
    const uint8_t *const p = tile + at + q * (16 * BN * 2);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4 *)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4 *)(p + 4 * BN * 2));
    const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
    return __builtin_bit_cast(bf16x8, u32x4{l[0], l[1], h[0], h[1]});
}

// What a lane needs of a tile, fixed for the whole reduction, and how far the
// loads have come.
struct Ctx {
    uint8_t *ring, *tiles;
    uint32_t aoff[2];
    int ac[2];                    // each A chunk's first n in its stage
    const uint8_t *A;             // of the next stage, wave-uniform
    const uint8_t *codes, *scales;  // this thread's block in weight row 0 of its projection
    int64_t crow, srow;           // bytes of a weight row
    int seg, c0;                  // projection and first weight row of the next stage
    int wave, lane, row, blk;     // this thread's weight row of a stage and block
};

// A thread's block of codes of one stage and its scale (a row past the last: zeros).
template <int FMT>
struct Raw {
    uint32_t c[(FMT == QL_FMT_INT8 ? 32 : 16) / 4];
    float s;
};

template <int FMT>
__device__ inline void start_segment(const DxArgs &a, Ctx &c, int m0, int k0)
{
    c.A = reinterpret_cast<const uint8_t *>(a.d[c.seg] + (int64_t)m0 * a.N + c.c0);
    // (blocks past K repeat the row's last one: those columns are not stored)
    const int b = min(k0 / 32 + c.blk, a.K / 32 - 1);
    c.codes = a.codes[c.seg] + (int64_t)b * (FMT == QL_FMT_INT8 ? 32 : 16);
    c.scales = static_cast<const uint8_t *>(a.scales[c.seg]) +
               (FMT == QL_FMT_MXFP4 ? b & ~3 : 2 * (b & ~1));
}

template <int FMT, int MS>
__device__ inline void issue(const DxArgs &a, Ctx &c, int m0, int k0, int slot)
{
    using G = Geo<FMT, MS>;
    const uint32_t base = dma_lds(c.ring + slot * G::STAGE);
    if (c.c0 + BC <= a.N) {
#pragma unroll
        for (int i = 0; i < G::ALOADS; ++i)
            dma_load16(c.A, c.aoff[i], base + (i * THREADS + c.wave * 64) * 16);
    } else {
#pragma unroll
        for (int i = 0; i < G::ALOADS; ++i)
            dma_load16_at(c.c0 + c.ac[i] < a.N ? c.A + c.aoff[i] : (const uint8_t *)zeros,
                          base + (i * THREADS + c.wave * 64) * 16);
    }
    // (rows past N repeat the last one, and are converted to zeros)
    const int64_t n = min(c.c0 + c.row, a.N - 1);
#pragma unroll
    for (int h = 0; h < G::CLOADS; ++h)
        dma_load16_at(c.codes + n * c.crow + 16 * h,
                      base + G::ABYTES + (h * THREADS + c.wave * 64) * 16);
    dma_load4_at(c.scales + n * c.srow, base + G::ABYTES + G::CBYTES + c.wave * 256);
    c.c0 += BC;
    c.A += BC * 2;
    if (c.c0 >= a.N && c.seg == 0) {
        c.seg = 1;
        c.c0 = 0;
        start_segment<FMT>(a, c, m0, k0);
    }
}

// step s of the whole reduction: first weight row in its projection
__device__ inline int first_row(int s, int seg_steps) { return (s >= seg_steps ? s - seg_steps : s) * BC; }

template <int FMT, int MS>
__device__ inline void read_raw(const Ctx &c, const uint8_t *st, int b, int n0, int N, Raw<FMT> &r)
{
    using G = Geo<FMT, MS>;
    const int tid = c.wave * 64 + c.lane;
    const bool in = n0 + c.row < N;
#pragma unroll
    for (int h = 0; h < G::CLOADS; ++h) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(st + G::ABYTES + (h * THREADS + tid) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            r.c[4 * h + e] = in ? v[e] : 0u;
    }
    const uint32_t d = *reinterpret_cast<const uint32_t *>(st + G::ABYTES + G::CBYTES + tid * 4);
    if constexpr (FMT == QL_FMT_MXFP4)
        r.s = mx_scale(d >> (8 * (b & 3)) & 255u);
    else
        r.s = plane_scale((float)__builtin_bit_cast(_Float16, (uint16_t)(d >> (16 * (b & 1)))));
    r.s = in ? r.s : 1.0f;
}

// a thread's converted chunk w in a weight tile
__device__ inline uint32_t w_at(const Ctx &c, int w)
{
    const int chunk = 4 * c.blk + w;
    return (uint32_t)(c.row * (BN * 2) + (chunk ^ bswz(c.row, chunk)) * 16);
}

template <int FMT, int MS>
__global__ __launch_bounds__(THREADS, WGS<FMT>) void gemm_dx_kernel(const DxArgs a)
{
    using G = Geo<FMT, MS>;
    constexpr int NST = G::NST, P = G::PLANES, KK = MS * NS * P, BM = G::BM, GROUP_M = 16 / MS;
    __shared__ __align__(16) uint8_t lds[G::LDS];
    const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.K + BN - 1) / BN;
    // each XCD takes a contiguous range of the tiles, in groups of 4 row tiles
    // walked row tile fastest; the parts of a tile are adjacent
    const int p = (int)blockIdx.x, grid = (int)gridDim.x;
    const int gq = grid >> 3, gr = grid & 7, xcd = p & 7, idx = p >> 3;
    const int local = xcd < gr ? xcd * (gq + 1) + idx : gr * (gq + 1) + (xcd - gr) * gq + idx;
    const int part = local % a.parts, tile = local / a.parts;
    const int gid = tile / (GROUP_M * tiles_n), within = tile - gid * (GROUP_M * tiles_n);
    const int gsz = min(tiles_m - gid * GROUP_M, GROUP_M);
    const int m0 = (gid * GROUP_M + within % gsz) * BM, k0 = within / gsz * BN;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;

    const int seg_steps = (a.N + BC - 1) / BC, all_steps = 2 * seg_steps;
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
        Ctx c;
        c.ring = lds + 2 * P * G::BTILE;
        c.tiles = lds;
        c.wave = wave;
        c.lane = lane;
        c.row = tid >> 3;
        c.blk = tid & 7;
        const int blk = min(k0 / 32 + c.blk, a.K / 32 - 1);
#pragma unroll
        for (int i = 0; i < G::ALOADS; ++i) {
            const int at = i * THREADS + tid, row = at >> 2, lc = (at & 3) ^ aswz(row);
            c.ac[i] = lc * 8;
            c.aoff[i] = (uint32_t)((min(m0 + row, a.M - 1) - m0) * (int64_t)a.N * 2 + lc * 16);
        }
        c.crow = (int64_t)(a.K / 32) * G::CODES;
        c.srow = (int64_t)(a.K / 32) * (FMT == QL_FMT_MXFP4 ? 1 : 2);
        c.seg = s0 >= seg_steps;
        c.c0 = first_row(s0, seg_steps);
        start_segment<FMT>(a, c, m0, k0);
#pragma unroll 1
        for (int t = 0; t < NST && t < ns; ++t)
            issue<FMT, MS>(a, c, m0, k0, t);

        // stage 0 converted, its first chunk's fragments and stage 1's codes in
        // registers
        Raw<FMT> raw;
        dma_wait<G::LOADS, NST - 1>(min(ns, NST) - 1);
        read_raw<FMT, MS>(c, c.ring, blk, first_row(s0, seg_steps), a.N, raw);
        uint32_t wat[4], aat[2], bat[NS];
#pragma unroll
        for (int w = 0; w < 4; ++w)
            wat[w] = w_at(c, w);
#pragma unroll
        for (int q = 0; q < 2; ++q)
            aat[q] = a_at(lane, q);
#pragma unroll
        for (int j = 0; j < NS; ++j)
            bat[j] = b_at(lane, wave * 64 + 32 * j);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            u32x4 hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t h, l;
                decode_word<FMT>(raw.c, 4 * w + e, raw.s, h, l);
                hi[e] = h;
                lo[e] = l;
            }
            *reinterpret_cast<u32x4 *>(c.tiles + wat[w]) = hi;
            if constexpr (P == 2)
                *reinterpret_cast<u32x4 *>(c.tiles + G::BTILE + wat[w]) = lo;
        }
        if (ns > 1) {
            dma_wait<G::LOADS, NST - 2>(min(ns, NST) - 2);
            read_raw<FMT, MS>(c, c.ring + G::STAGE, blk, first_row(s0 + 1, seg_steps), a.N, raw);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");  // (no read of the stage before the barrier)
        bf16x8 av[MS], bv[P][NS];
#pragma unroll
        for (int v = 0; v < P; ++v)
#pragma unroll
            for (int j = 0; j < NS; ++j)
                bv[v][j] = read_b(c.tiles + v * G::BTILE, bat[j], 0);
#pragma unroll
        for (int i = 0; i < MS; ++i)
            av[i] = read_a(c.ring, aat[0], i);

        int slot = 0, slot2 = 2 % NST;  // of stages t and t + 2
        for (int t = 0; t < ns; ++t) {
            const uint8_t *const cur = c.ring + slot * G::STAGE;
            const int nslot = slot + 1 == NST ? 0 : slot + 1;
            const uint8_t *const btile = c.tiles + (t & 1) * (P * G::BTILE);
            uint8_t *const bnext = c.tiles + ((t + 1) & 1) * (P * G::BTILE);
            bf16x8 an[MS], bn[P][NS];
            // chunk 0; behind its MFMAs the fragments of chunk 1 and stage t + 1's
            // weights (after the last stage: converted from old codes, never
            // multiplied)
            u32x4 hi, lo;
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const int v = P - 1 - k / (MS * NS), i = k / NS % MS, j = k % NS;
                acc[i][j] =
                    __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[i], bv[v][j], acc[i][j], 0, 0, 0);
                // (reads first, two fragments at a time: they have to be there by the
                // chunk's end)
                if (k < P * NS / 2) {
                    bn[k / (NS / 2)][0] = read_b(btile + k * G::BTILE, bat[0], 1);
                    bn[k / (NS / 2)][1] = read_b(btile + k * G::BTILE, bat[1], 1);
                } else if (k < P * NS / 2 + MS / 2) {
                    an[2 * k - P * NS] = read_a(cur, aat[1], 2 * k - P * NS);
                    an[2 * k - P * NS + 1] = read_a(cur, aat[1], 2 * k - P * NS + 1);
                }
#pragma unroll
                for (int w = k * 16 / KK; w < (k + 1) * 16 / KK; ++w) {
                    uint32_t h, l;
                    decode_word<FMT>(raw.c, w, raw.s, h, l);
                    dma_pin(h);
                    hi[w & 3] = h;
                    if constexpr (P == 2) {
                        dma_pin(l);
                        lo[w & 3] = l;
                    }
                    if ((w & 3) == 3) {
                        *reinterpret_cast<u32x4 *>(bnext + wat[w >> 2]) = hi;
                        if constexpr (P == 2)
                            *reinterpret_cast<u32x4 *>(bnext + G::BTILE + wat[w >> 2]) = lo;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // the stage is in registers, the next one's weights are written and (its
            // loads came with theirs) its dG has landed
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (t + NST < ns)
                issue<FMT, MS>(a, c, m0, k0, slot);
            // stage t + 2 has landed where only those younger are in flight
            if (t + NST < ns)
                __builtin_amdgcn_s_waitcnt(dma_vmcnt((NST - 2) * G::LOADS));
            else if (t + 2 < ns)
                dma_wait<G::LOADS, NST - 2>(ns - 3 - t);
            read_raw<FMT, MS>(c, c.ring + slot2 * G::STAGE, blk, first_row(s0 + t + 2, seg_steps), a.N,
                          raw);
            // chunk 1; behind its MFMAs stage t + 1's first fragments
            bf16x8 a0[MS], b0[P][NS];
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const int v = P - 1 - k / (MS * NS), i = k / NS % MS, j = k % NS;
                acc[i][j] =
                    __builtin_amdgcn_mfma_f32_32x32x16_bf16(an[i], bn[v][j], acc[i][j], 0, 0, 0);
                if (k < P * NS / 2) {
                    b0[k / (NS / 2)][0] = read_b(bnext + k * G::BTILE, bat[0], 0);
                    b0[k / (NS / 2)][1] = read_b(bnext + k * G::BTILE, bat[1], 0);
                } else if (k < P * NS / 2 + MS / 2) {
                    const uint8_t *const st = c.ring + nslot * G::STAGE;
                    a0[2 * k - P * NS] = read_a(st, aat[0], 2 * k - P * NS);
                    a0[2 * k - P * NS + 1] = read_a(st, aat[0], 2 * k - P * NS + 1);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < MS; ++i)
                av[i] = a0[i];
#pragma unroll
            for (int v = 0; v < P; ++v)
#pragma unroll
                for (int j = 0; j < NS; ++j)
                    bv[v][j] = b0[v][j];
            slot = nslot;
            slot2 = slot2 + 1 == NST ? 0 : slot2 + 1;
        }
    }
    __syncthreads();  // LDS is free: the 32 x 32 tiles turn through patches of it

    const bool to_part = a.parts > 1;
    Epilogue e{};
    e.ybf16 = !to_part && a.outbf16;
    float *const Y = to_part ? a.part + (int64_t)part * a.M * a.K : static_cast<float *>(a.out);
    // (K % 32 == 0 and aligned outputs: whole groups of four)
    strip_store<false>(e, Y, a.M, a.K, m0, k0 + wave * 64,
                       reinterpret_cast<float *>(lds) + wave * STRIP_PATCH, lane, acc, true,
                       !to_part);
}

}  // namespace

bool dx_takes(int64_t K, const void *scales0, const void *scales1)
{
    return K % 128 == 0 && ((uintptr_t)scales0 & 3) == 0 && ((uintptr_t)scales1 & 3) == 0;
}

hipError_t launch_gemm_dx(int fmt, const DxArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(gemm_tiles(a.rows, a.M, a.K) * a.parts)), block(THREADS);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    auto with = [&](auto fmtc) {
        constexpr int F = decltype(fmtc)::value;
        a.rows == 64 ? go(gemm_dx_kernel<F, 2>) : go(gemm_dx_kernel<F, 4>);
    };
    if (fmt == QL_FMT_MXFP4)
        with(std::integral_constant<int, QL_FMT_MXFP4>{});
    else if (fmt == QL_FMT_Q4)
        with(std::integral_constant<int, QL_FMT_Q4>{});
    else
        with(std::integral_constant<int, QL_FMT_INT8>{});
    return hipGetLastError();
}

}  // namespace qlk
