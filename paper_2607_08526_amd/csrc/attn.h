// What the masked attention's forward (attn_forward.hip) and backward kernels
// (attn_backward.hip) share: where a sequence's rows lie, tiles of rows in LDS, and the
// operands of the matrix instructions.
#pragma once

#include "dma.h"
#include "internal.h"

namespace qlk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// two fp32 values rounded to nearest even bf16, packed
__device__ inline uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}

// One side (queries or keys) of sequence b: its first row, its live rows, and the rows
// of its place (those past the live ones are padding).
struct SeqRows {
    int64_t first;
    int len, cap;
};

// Offsets and lengths are the caller's device data: whatever they hold, the rows stay
// inside the tensor and no sequence has more than T.
__device__ inline SeqRows seq_rows(const int64_t *off, const int64_t *lens, int64_t rows, int T,
                                   int b)
{
    SeqRows s;
    s.first = (int64_t)b * T;
    s.cap = T;
    if (off) {
        const int64_t lo = off[b] < 0 ? 0 : off[b] > rows ? rows : off[b];
        const int64_t hi = off[b + 1] < lo ? lo : off[b + 1] > rows ? rows : off[b + 1];
        s.first = lo;
        s.cap = hi - lo < T ? (int)(hi - lo) : T;
    }
    s.len = s.cap;
    if (lens)
        s.len = lens[b] < 0 ? 0 : lens[b] > s.cap ? s.cap : (int)lens[b];
    return s;
}

// LDS tiles hold rows of D channels as they come, in chunks of 16 bytes; chunk c of
// row r is kept at place c ^ swz(r), so that both ways in which a tile is read spread
// over the banks (64 of 4 bytes): 16 rows' equal chunks (rows of an operand), and four
// consecutive rows' four neighbouring chunks (transposed).  D = 64: a row is half the
// banks, so rows of one parity need eight places, rows r and r + 2 unlike halves of them;
// D = 128: 16 rows need 16 places, four consecutive ones unlike quarters.
template <int D>
__device__ inline int swz(int r)
{
    if constexpr (D == 64)
        return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1 | ((r >> 3) & 1);
    else
        return (r & 3) << 2 | ((r >> 2) & 3);
}

// Operand of 32 rows of a tile, 8 channels from 16 s + 8 hf on a lane (row l32 of them)
template <int D>
__device__ inline bf16x8 row_operand(const uint8_t *tile, int row, int s, int hf)
{
    return __builtin_bit_cast(
        bf16x8, *reinterpret_cast<const u32x4 *>(tile + row * (2 * D) +
                                                 ((2 * s + hf) ^ swz<D>(row)) * 16));
}

// Operand of 32 channels from 32 t on, transposed: lane l has channel 32 t + l % 32 of
// the 8 rows {16 c + 4 h + i, 16 c + 8 + 4 h + i : i < 4}, h = l / 32 (the order in
// which the accumulators of a 32 x 32 product hold their rows), by the transposing LDS
// read: within each group of 16 lanes, result lane 4 q + p receives element p of the 8
// bytes that source lanes q, 4 + q, 8 + q and 12 + q address.
template <int D>
__device__ inline bf16x8 transposed_operand(const uint8_t *tile, int c, int t, int lane)
{
    const int row0 = 16 * c + 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int unit = 8 * t + 4 * ((lane >> 4) & 1) + (lane & 3);  // of 8 bytes
    u32x2 v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int row = row0 + 8 * u;
        const uint32_t off = row * (2 * D) + (((unit >> 1) ^ swz<D>(row)) * 16) + (unit & 1) * 8;
        v[u] = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4 *)(tile + off)));
    }
    return __builtin_bit_cast(bf16x8, u32x4{v[0][0], v[0][1], v[1][0], v[1][1]});
}

__device__ inline f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Loads of a tile of ROWS rows by T threads: slot i = j T + t of 16 bytes for thread t's
// load j is row i / (D / 8), place i % (D / 8).
template <int D, int ROWS, int T>
struct TileLoad {
    static constexpr int CH = D / 8, N = ROWS * CH / T;
    static_assert(N >= 1 && ROWS * CH % T == 0, "");
    uint32_t full[N];

    // offsets from the tile's first row (ld: elements of a row, fewer than 2^24)
    __device__ inline void init(int64_t ld, int tid)
    {
#pragma unroll
        for (int j = 0; j < N; ++j)
            full[j] = offset(j, ROWS, ld, tid);
    }
    __device__ static inline uint32_t offset(int j, int rows, int64_t ld, int tid)
    {
        const int i = j * T + tid, r = i / CH, lc = (i % CH) ^ swz<D>(r);
        return (uint32_t)(min(r, rows - 1) * (int)ld + 8 * lc) * 2u;
    }
    // rows: those there are (>= 1); the tile's others repeat the last of them
    __device__ inline void issue(const uint8_t *first, int rows, int64_t ld, const uint8_t *lds,
                                 int tid) const
    {
        const uint32_t at = dma_lds(lds) + (tid & ~63) * 16;
        if (rows >= ROWS) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                dma_load16(first, full[j], at + j * T * 16);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                dma_load16(first, offset(j, rows, ld, tid), at + j * T * 16);
        }
    }
};

template <bool B>
struct Flag {
    static constexpr bool value = B;
};
template <int I>
struct Index {
    static constexpr int value = I;
};

// f(Index<0>), f(Index<1>), ..., f(Index<N - 1>)
template <int N, int I = 0, typename F>
__device__ inline void each(F &&f)
{
    if constexpr (I < N) {
        f(Index<I>{});
        each<N, I + 1>(f);
    }
}

// x of lanes l and l ^ 32, in this order for both
__device__ inline void both_halves(float x, float &lo, float &hi)
{
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    lo = __uint_as_float(r[0]);
    hi = __uint_as_float(r[1]);
}

// The order of instructions stays as written across this point.
__device__ inline void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// What a workgroup does: part `part` of block `blk` of rows (0: the longest of causal ones)
// of key head and sequence `unit`.
struct Work {
    int part, blk, unit;
};

// Workgroup p runs on XCD p % 8: each XCD takes a contiguous range of the grid's work,
// so that the tiles which several workgroups read come into one L2 (sequences vary fastest
// in it: each XCD has long and short ones.  Five packed clips of 387 to 645 tokens, 32
// heads: with heads fastest the XCD of the longest has 1.5 times the work of the
// average).  Causal blocks, long and short: see order_work.
__host__ __device__ inline Work work_of(const SeqAttn &s, int p, int grid, int parts, int nb)
{
    const int q = grid >> 3, r = grid & 7, xcd = p & 7, i = p >> 3;
    const int n = xcd < r ? q + 1 : q, first = xcd < r ? xcd * n : r * (q + 1) + (xcd - r) * q;
    const int half = (n + 1) / 2;
    const int L = first + (s.fold && i >= half ? n - 1 - (i - half) : i);
    Work w;
    int at = L / parts;
    w.part = L - at * parts;
    w.unit = at / nb;
    w.blk = at - w.unit * nb;
    if (s.group > 1) {
        const int units = s.B * s.Hk / 8;  // of an XCD: first to first + units - 1
        const int u0 = w.unit / units * units, g0 = (w.unit - u0) / s.group * s.group;
        const int size = s.group < units - g0 ? s.group : units - g0;
        at -= (u0 + g0) * nb;
        w.blk = at / size;
        w.unit = u0 + g0 + at - w.blk * size;
    }
    return w;
}

// The order of a launch of `blocks` workgroups for each of the B Hk units, `resident` of
// them on a CU at a time.  Causal blocks take from next to nothing to twice the average.
// Where all run at once, two on a CU, the second half of an XCD's range is taken from its
// end: a CU's two are a long and a short one.  Where they do not, a unit's longest come
// first, and the places that its short ones leave early take the next unit's long ones;
// units that do not fill an XCD's places twice are taken together, as many as do, their
// longest first.  4096 queries of 32 heads of 64, us forward, dq, dk and dv: 122 / 151 / 192
// unit by unit, 108 / 134 / 167 four together; 2 sequences of 2048, 8 heads of 128 with 4
// query heads each, dk and dv in 2 parts: 194 and, two together, 184.  (One workgroup on a
// CU at a time, so nothing taken from the end: dk and dv of one such sequence 104, not 124.)
inline void order_work(SeqAttn &s, int64_t blocks, int resident)
{
    const int64_t units = (int64_t)s.B * s.Hk, places = (int64_t)resident * s.cus / 8;
    s.fold = s.causal && resident == 2 && blocks * units <= 8 * places;
    s.group = 1;
    if (s.causal && !s.fold && units % 8 == 0 && blocks > 0)
        s.group = (int)((2 * places + blocks - 1) / blocks);
}

}  // namespace qlk
