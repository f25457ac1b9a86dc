// The masked attention's backward pass.  With P_ij = exp(s_ij - lse_i) formed again from
// the forward's lse (the probabilities are never kept) and d_i = <dO_i, O_i>,
//
//   dV_j = sum_i P_ij dO_i,  dP_ij = <dO_i, V_j>,  dS_ij = P_ij (dP_ij - d_i),
//   dQ_i = scale sum_j dS_ij K_j,  dK_j = scale sum_i dS_ij Q_i
//
// Two launches of one kernel, so that every sum has one order (no atomics): the first
// keeps rows of queries and streams keys past them (dQ; it also leaves lse log2(e) and d
// for the second), the second keeps keys and streams queries (dK, dV).  Both form P and
// dP: 7 products of dh flops per pair instead of 5.
//
// A wavefront keeps 32 rows of two tensors in registers as right operands (Q, dO; or K,
// V); tiles of BT rows of the other two (K, V; or Q, dO) come into LDS by direct loads, a
// ring of BUFS of them, and are taken in blocks of 32 rows.  S and dP of a block are
// formed with the streamed rows as left operand: a lane then holds 16 streamed rows of one
// kept row, just what the right operand of the second products (transposed left operand:
// dQ^T += K^T dS^T, dV^T += dO^T P, dK^T += Q^T dS) wants of P and dS, which are rounded to
// bf16 for it.  Matrix and vector units run beside each other within a wavefront: P and dS
// of block i are formed between the matrix instructions of block i + 1's S and dP; block
// i's second products follow.
//
// What is rounded to bf16, and why: P and dS, as the matrix instructions take them (fp32
// would take 16 times as long; two bf16 each, as for few rows, 10 products for 7); d is as
// exact as the caller's O.  What d is off by counts times sum P K in dq, which with its other
// roundings is off by 0.0025 of its norm for scores of a spread of 1 and either O; at a spread
// of 10 by 0.0059 with a bf16 O and 0.0034 with an fp32 one.  d could be made exact from this kernel's own sums (the rest that a row's
// dS leave, 0 in exact arithmetic), but dq's correction takes sum P K: a fourth product
// beside three (dS as two bf16 is one: 128 queries over 4096 keys, 4 sequences of 32 heads
// of 64, 50 us for 43) and D x 32 more accumulators, for every caller, where an fp32 O costs
// its bytes.
//
// What bounds it, measured in us, dq / dk and dv: 4096 queries and keys of 32 heads of 64
// 215 / 270, of 16 heads of 128 199 / 285: 960 to 1040 TFLOP/s of dq's three products and
// the four of dk and dv.  Matrix cores are busy in 0.5 (dq) and 0.6 of a CU's cycles, vector
// instructions in 0.6, and the clock falls as these shares rise.  One causal sequence of
// 2048, 8 key heads of 128 with 4 query heads each: 77 / 100 and 12 for adding up 4 parts,
// where half of the time without a mask is 55 / 75 and 8: a grid that the GPU holds at once,
// as forward.  Five packed sequences of 387 to 645, 32 heads of 64: 44 / 52, launches of 960
// workgroups for 512 places, of 7 to 11 tiles each: their first loads and last stores weigh
// as much as a third of these.
//
// Both launches in one, or one that adds dq up by atomics, would save two of seven products;
// the one needs the registers of both (two accumulators of D x 32 more), the other gives
// sums whose order changes.
#include <algorithm>
#include <cmath>

#include "attn.h"

namespace qlk {
namespace {

constexpr int THREADS = 256;
constexpr float LOG2E = 1.44269504088896340736f;

constexpr int KEEP = 128;  // kept rows of a workgroup
// Where a workgroup streams at most so many rows, its sums, of few terms each, take what
// rounding averages out in longer ones: P and dS enter the products as two bf16, 16 bits of
// them, and d_i is formed as sum P_ij dP_ij in a pass of its own, not from a bf16 O.  Tiles
// are loaded a ring at a time and nothing overlaps (107 queries and keys of 48 heads of 64: dk
// and dv in 10.1 us, 8.2 with P and dS as one bf16 each and overlapped; dq 10.3 and 10.7).
// (With one bf16 each, dq at 2 to 3 keys was off by 0.0027 to 0.0030 of its norm, where the
// output's own rounding is 0.0017.)
constexpr int FEW = 128;

// The same where the outputs have few rows, of all sequences and heads together (TWO): their
// roundings do not average out over the output either (dq of one query over 479 keys, 4
// heads of 4 sequences, was off by 0.0025 of its norm; 0.0017 so).  The tiles overlap as in
// longer outputs, and each second product is taken twice: in launches that leave most CUs
// idle.  (us, as one and as two bf16: dq of 5 queries over 3000 keys, 2 heads of 64 10.7 and
// 11.3, of one over 8192, 8 sequences of 32 heads of 128 on 8 63 and 72; dk and dv of 8 keys
// under 700 queries of 8 heads of 128 on one 21.0 and 24.2.)
constexpr int FEW_OUT = 2048;
template <int D, bool KEYS, int BT, int BUFS, bool TWO>
__global__ __launch_bounds__(THREADS)
__attribute__((amdgpu_waves_per_eu(D == 128 && (KEYS || TWO) ? 1 : 2, 2)))
void seq_attn_grad_kernel(const SeqAttnGrad a)
{
    constexpr int TILE = BT * D * 2;  // bytes of a tile
    constexpr int DT = D / 32, DS = D / 16, SUB = BT / 32;
    constexpr int BUF = 2 * TILE + (KEYS ? 1024 : 0);  // (the sums of 64 rows)
    __shared__ __align__(16) uint8_t lds[BUFS * BUF + (KEYS ? 16 : 0)];
    uint8_t *const zeros = lds + BUFS * BUF;
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hf = lane >> 5;

    const SeqAttn &s = a.s;
    const int G = s.H / s.Hk, parts = KEYS ? a.kparts : a.qparts;
    const int rows = KEYS ? s.KT : s.T * G;  // kept, of a (sequence, key head)
    const int nb = (rows + KEEP - 1) / KEEP;
    const Work w = work_of(s, (int)blockIdx.x, (int)gridDim.x, parts, nb);
    const int part = w.part, unit = w.unit, hk = unit / s.B, b = unit - hk * s.B;
    // (the longest of causal blocks: the last queries, the first keys)
    const int blk = s.causal && !KEYS ? nb - 1 - w.blk : w.blk;
    const SeqRows Q = seq_rows(s.q_off, s.q_len, s.qrows, s.T, b);
    const SeqRows K = seq_rows(s.k_off, s.k_len, s.krows, s.KT, b);
    const int row0 = blk * KEEP;
    if (row0 >= (KEYS ? K.cap : Q.cap * G))
        return;
    const int shift = K.len - Q.len;  // causal: query t sees the keys up to t + shift
    const float c = s.c;

    const int wrow = row0 + wave * 32;  // the wavefront's first row
    // tiles [first, first + tiles) of streamed rows, for keys of each head in turn
    int first = 0, tiles;
    if (KEYS) {
        first = s.causal ? max(0, row0 - shift) / BT : 0;
        tiles = row0 < K.len ? max(0, (Q.len + BT - 1) / BT - first) : 0;
    } else {
        const int tmax = min((row0 + KEEP - 1) / G, Q.len - 1);
        const int keys = Q.len > row0 / G
                             ? max(0, (s.causal ? min(K.len - 1, tmax + shift) : K.len - 1) + 1)
                             : 0;
        tiles = (keys + BT - 1) / BT;
    }
    const int64_t all = (int64_t)tiles * (KEYS ? G : 1);
    const int j0 = (int)(all * part / parts), j1 = (int)(all * (part + 1) / parts);
    // streamed rows that need no mask
    const int free_lo = KEYS && s.causal ? wrow + 31 - shift : 0;
    const int free_hi = KEYS ? Q.len - 1
                             : (s.causal ? min(K.len - 1, wrow / G + shift) : K.len - 1);

    const int64_t ld1 = KEYS ? s.ldq : s.ldk, ld2 = KEYS ? a.lddo : s.ldv;
    TileLoad<D, BT, THREADS> load1, load2;
    load1.init(ld1, tid);
    load2.init(ld2, tid);
    constexpr int LOADS = 2 * TileLoad<D, BT, THREADS>::N + (KEYS ? 1 : 0);  // a tile's
    // The tile that is loaded next: tile ft of head fh, its rows' first bytes and number,
    // and its buffer.  (Counted on from tile to tile: scalar instructions take their turn
    // with the others of a wavefront, a division and four products a tile among them.)
    int ft, fh, fleft, fbuf = 0;
    const uint8_t *f1, *f2;
    const float *fsums;
    auto aim = [&](int j) {
        const int g = KEYS ? j / tiles : 0;
        ft = j - g * tiles;
        fh = KEYS ? hk * G + g : hk;
        const int64_t at = (KEYS ? Q.first : K.first) + (first + ft) * BT;
        fleft = (KEYS ? Q.len : K.len) - (first + ft) * BT;
        f1 = reinterpret_cast<const uint8_t *>((KEYS ? s.q : s.k) + at * ld1 + fh * D);
        f2 = reinterpret_cast<const uint8_t *>((KEYS ? a.dO : s.v) + at * ld2 + fh * D);
        fsums = a.sums + (fh * s.qrows + at) * 4;
    };
    auto following = [](int buf) { return buf == (BUFS - 1) * BUF ? 0 : buf + BUF; };
    auto fetch = [&] {
        const uint8_t *const buf = lds + fbuf;
        load1.issue(f1, fleft, ld1, buf, tid);
        load2.issue(f2, fleft, ld2, buf + TILE, tid);
        if (KEYS)  // (every wavefront the same: all have as many loads in flight)
            dma_load16(fsums, min(lane, fleft - 1) * 16, dma_lds(buf + 2 * TILE));
        fbuf = following(fbuf);
        ++ft;
        if (KEYS && ft == tiles) {
            aim((fh - hk * G + 1) * tiles);
        } else {
            f1 += BT * 2 * ld1;
            f2 += BT * 2 * ld2;
            fsums += BT * 4;
            fleft -= BT;
        }
    };

    // The first tiles, before the kept rows (whose loads they pass on the way); where they
    // are few, all (of dq those of other parts too: d is a sum over them)
    static_assert(KEYS || FEW / BT <= BUFS, "");
    const bool few = (KEYS ? (int64_t)(Q.len - first * BT) * G : tiles * BT) <= FEW;
    const int l0 = few && !KEYS ? 0 : j0;
    const int l1 = few && !KEYS ? tiles : min(j1, j0 + (few ? BUFS : BUFS - 1));
    if (l0 < l1) {
        aim(l0);
        for (int j = l0; j < l1; ++j)
            fetch();
    }

    // the kept row of this lane: its operands, and the streamed rows lo to hi that meet it
    const int row = wrow + l32;
    const int t = KEYS ? row : row / G, head = KEYS ? hk : hk * G + row - t * G;
    const bool live = t < (KEYS ? K.len : Q.len);
    bf16x8 x1[DS], x2[DS];
    {
        const uint16_t *p1 = KEYS ? s.k + (K.first + t) * s.ldk : s.q + (Q.first + t) * s.ldq;
        const uint16_t *p2 = KEYS ? s.v + (K.first + t) * s.ldv : a.dO + (Q.first + t) * a.lddo;
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            u32x4 v1 = {0u, 0u, 0u, 0u}, v2 = v1;
            if (live) {
                v1 = *reinterpret_cast<const u32x4 *>(p1 + head * D + 16 * i + 8 * hf);
                v2 = *reinterpret_cast<const u32x4 *>(p2 + head * D + 16 * i + 8 * hf);
            }
            x1[i] = __builtin_bit_cast(bf16x8, v1);
            x2[i] = __builtin_bit_cast(bf16x8, v2);
        }
    }
    const int lo = KEYS && s.causal ? t - shift : 0;
    const int hi = !live ? -1 : KEYS ? Q.len - 1 : s.causal ? min(K.len - 1, t + shift) : K.len - 1;
    // of a kept query: lse in powers of two, and d = sum dO O
    float lse2 = INFINITY, delta = 0.0f;
    if (!KEYS && live) {
        const int64_t at = (Q.first + t) * a.ldo + head * D + 8 * hf;
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            float o[8];
            if (a.obf16) {
                const uint16_t *p = static_cast<const uint16_t *>(a.o) + at + 16 * i;
                const u32x2 w[2] = {*reinterpret_cast<const u32x2 *>(p),
                                    *reinterpret_cast<const u32x2 *>(p + 4)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o[2 * j] = __uint_as_float(w[j >> 1][j & 1] << 16);
                    o[2 * j + 1] = __uint_as_float(w[j >> 1][j & 1] & 0xFFFF0000u);
                }
            } else {
                const float *p = static_cast<const float *>(a.o) + at + 16 * i;
                const f32x4_t w[2] = {*reinterpret_cast<const f32x4_t *>(p),
                                      *reinterpret_cast<const f32x4_t *>(p + 4)};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    o[j] = w[j >> 2][j & 3];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                delta = __builtin_fmaf((float)x2[i][j], o[j], delta);
        }
        const float l = a.lse[head * s.qrows + Q.first + t];
        lse2 = l == -INFINITY ? INFINITY : l * LOG2E;
    }
    auto halves = [](float x) {
        float l, h;
        both_halves(x, l, h);
        return l + h;
    };
    if (!KEYS)
        delta = halves(delta);
    f32x16 acc1[DT], acc2[KEYS ? DT : 1];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            acc1[d][r] = 0.0f;
            if (KEYS)
                acc2[d][r] = 0.0f;
        }

    // What a tile's products leave: its scores and dP, then P and dS as operands.
    struct Raw {
        f32x16 s, dp;
    };
    struct Cooked {
        bf16x8 p[KEYS ? 2 : 1], ds[2];
    };
    // Values 2 I and 2 I + 1 of a lane: streamed rows r0 + 8 (r / 4) + 4 hf + r % 4, r = 2 I
    // and 2 I + 1; from, to: lo and hi less r0 + 4 hf.
    auto probability = [&](auto maskc, auto ic, int from, int to, const Raw &x, float (&p)[2],
                           float (&ds)[2]) {
        constexpr bool MASK = decltype(maskc)::value;
        constexpr int I = decltype(ic)::value;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = 2 * I + k, at = 8 * (r >> 2) + (r & 3);
            p[k] = __builtin_amdgcn_exp2f(KEYS ? x.s[r] * c : __builtin_fmaf(x.s[r], c, -lse2));
            if (MASK)
                p[k] = at <= to && (!KEYS || at >= from) ? p[k] : 0.0f;
            ds[k] = p[k] * (KEYS ? x.dp[r] : x.dp[r] - delta);
        }
    };
    auto put = [](bf16x8 &v, int i, uint32_t w) {
        u32x4 u = __builtin_bit_cast(u32x4, v);
        u[i] = w;
        v = __builtin_bit_cast(bf16x8, u);
    };
    // (as two bf16 each with `two`: y and what it leaves)
    auto cook = [&](auto maskc, auto twoc, auto ic, int from, int to, const Raw &x, Cooked &y,
                    Cooked &rest) {
        constexpr int I = decltype(ic)::value;
        float p[2], ds[2];
        probability(maskc, ic, from, to, x, p, ds);
        if constexpr (!decltype(twoc)::value) {
            if constexpr (KEYS)
                put(y.p[I / 4], I % 4, pack_bf16(p[0], p[1]));
            put(y.ds[I / 4], I % 4, pack_bf16(ds[0], ds[1]));
            return;
        }
        auto split = [&](bf16x8 &v, bf16x8 &w, const float (&f)[2]) {
            const uint32_t hi = pack_bf16(f[0], f[1]);
            put(v, I % 4, hi);
            put(w, I % 4, pack_bf16(f[0] - __uint_as_float(hi << 16),
                                    f[1] - __uint_as_float(hi & 0xFFFF0000u)));
        };
        if constexpr (KEYS)
            split(y.p[I / 4], rest.p[I / 4], p);
        split(y.ds[I / 4], rest.ds[I / 4], ds);
    };
    // D = 128 (one code for every tile, or the accumulators' registers run out): the mask
    // is what a tile's scores start from, 0 or -infinity.
    constexpr bool BIAS = D == 128 || KEYS;
    auto bias = [&](int r0, Raw &x) {
        const int from = lo - r0 - 4 * hf, to = hi - r0 - 4 * hf;
        if (r0 >= free_lo && r0 + 31 <= free_hi) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                x.s[r] = 0.0f;
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int at = 8 * (r >> 2) + (r & 3);
                x.s[r] = at <= to && (!KEYS || at >= from) ? 0.0f : -INFINITY;
            }
        }
    };
    // The matrix instructions of a step: S and dP of the tile in next (for kept keys they
    // start with -lse / scale and -d of the streamed queries, three bf16 each that add up
    // to 24 bits: as products with ones, two matrix instructions and LDS reads a block, where
    // reading them in the accumulators' layout, 16 values a lane each, takes eight reads and
    // 32 registers; each with zeros beside it, not the other: a d that is not finite must not
    // reach P), then the second products of the tile in prev.
    constexpr int SUMS = KEYS ? 2 : 0, FIRST = SUMS + 2 * DS, SECOND = (KEYS ? 4 : 2) * DT;
    const uint32_t one = hf == 0 ? 0x3F80u : 0u, ones = one | one << 16;
    const bf16x8 ones3 = __builtin_bit_cast(bf16x8, u32x4{ones, one, 0u, 0u});
    // (block NS of the tile in next, block PS of that in prev)
    auto operand = [&](auto ic, auto nsc, auto psc, const uint8_t *next, const uint8_t *prev) {
        constexpr int I = decltype(ic)::value, NS = decltype(nsc)::value, PS = decltype(psc)::value;
        if constexpr (I < SUMS) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(
                hf ? zeros : next + 2 * TILE + 512 * NS + l32 * 16 + 8 * I);
            return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], 0u, 0u});
        } else if constexpr (I < FIRST) {
            return row_operand<D>(next + (I % 2) * TILE, 32 * NS + l32, (I - SUMS) / 2, hf);
        } else {
            constexpr int k = I - FIRST, which = KEYS ? k % 2 : 0, m = KEYS ? k / 2 : k;
            return transposed_operand<D>(prev + which * TILE, 2 * PS + m / DT, m % DT, lane);
        }
    };
    auto multiply = [&](auto twoc, auto ic, bf16x8 w, Raw &x, const Cooked &y,
                        const Cooked &rest) {
        constexpr int I = decltype(ic)::value;
        if constexpr (I < FIRST) {
            const f32x16 zero = {};
            constexpr int i = (I - SUMS) / 2;
            if constexpr (I % 2 == 0)
                x.s = mfma(w, I < SUMS ? ones3 : x1[I < SUMS ? 0 : i],
                           I == 0 && !BIAS ? zero : x.s);
            else
                x.dp = mfma(w, I < SUMS ? ones3 : x2[I < SUMS ? 0 : i], I == 1 ? zero : x.dp);
        } else {
            constexpr int k = I - FIRST, m = KEYS ? k / 2 : k;
            constexpr bool second = KEYS && k % 2;
            f32x16 &acc = second ? acc2[KEYS ? m % DT : 0] : acc1[m % DT];
            acc = mfma(w, second ? y.p[KEYS ? m / DT : 0] : y.ds[m / DT], acc);
            if constexpr (decltype(twoc)::value)
                acc = mfma(w, second ? rest.p[KEYS ? m / DT : 0] : rest.ds[m / DT], acc);
        }
    };
    // The first products of the next block with the PAIRS steps of cook for this one between
    // them, then this one's second products; operands are read AHEAD of their instruction.
    constexpr int AHEAD = 3, PAIRS = 8;
    auto run = [&](auto maskc, auto subc, const uint8_t *buf, const uint8_t *next, int r0,
                   const Raw &cur, Raw &nxt, Cooked &now, Cooked &rest) {
        constexpr auto ns = Index<(decltype(subc)::value + 1) % SUB>{};
        const int from = lo - r0 - 4 * hf, to = hi - r0 - 4 * hf;
        constexpr int N = FIRST + SECOND;
        bf16x8 w[AHEAD + 1];
        each<AHEAD>([&](auto ic) { w[decltype(ic)::value] = operand(ic, ns, subc, next, buf); });
        each<N>([&](auto ic) {
            constexpr int I = decltype(ic)::value;
            if constexpr (I + AHEAD < N)
                w[(I + AHEAD) % (AHEAD + 1)] =
                    operand(Index<I + AHEAD>{}, ns, subc, next, buf);
            multiply(Flag<TWO>{}, ic, w[I % (AHEAD + 1)], nxt, now, rest);
            if constexpr (I < FIRST) {
                constexpr int P0 = PAIRS * I / FIRST, P1 = PAIRS * (I + 1) / FIRST;
                each<P1 - P0>([&](auto pc) {
                    cook(maskc, Flag<TWO>{}, Index<P0 + decltype(pc)::value>{}, from, to, cur,
                         now, rest);
                });
                keep_order();
            }
        });
    };
    auto first_products = [&](auto subc, const uint8_t *buf, int r0, Raw &x) {
        if (BIAS)
            bias(r0, x);
        Cooked none;
        each<FIRST>([&](auto ic) {
            multiply(Flag<false>{}, ic, operand(ic, subc, subc, buf, buf), x, none, none);
        });
    };
    auto second_products = [&](auto twoc, auto subc, const uint8_t *buf, const Cooked &y,
                               const Cooked &rest) {
        Raw none;
        each<SECOND>([&](auto ic) {
            constexpr int I = FIRST + decltype(ic)::value;
            multiply(twoc, Index<I>{}, operand(Index<I>{}, subc, subc, buf, buf), none, y, rest);
        });
    };

    if (KEYS && tid == 0)
        *reinterpret_cast<u32x4 *>(zeros) = u32x4{0u, 0u, 0u, 0u};
    if (l0 < l1 && few) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    if constexpr (!KEYS) {
        if (few && tiles > 0) {
            float d = 0.0f;
            for (int j = 0; j < tiles; ++j)
                each<SUB>([&](auto subc) {
                    const int r0 = j * BT + 32 * decltype(subc)::value;
                    Raw x;
                    first_products(subc, lds + j * BUF, r0, x);
                    const int to = hi - r0 - 4 * hf;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x.s[r], c, -lse2));
                        if (8 * (r >> 2) + (r & 3) <= to)
                            d = __builtin_fmaf(p, x.dp[r], d);
                    }
                });
            delta = halves(d);
        }
        if (live && part == 0 && hf == 0) {
            // -lse / scale and -d as three bf16 each (a query that sees no key: so low that
            // its probabilities are 0)
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = i ? -delta : lse2 == INFINITY ? -1e38f : -lse2 / c;
                uint32_t part3[3];
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    part3[k] = pack_bf16(x, 0.0f);
                    x -= __uint_as_float(part3[k] << 16);
                }
                w[2 * i] = part3[0] | part3[1] << 16;
                w[2 * i + 1] = part3[2];
            }
            *reinterpret_cast<u32x4 *>(a.sums + (head * s.qrows + Q.first + t) * 4) =
                u32x4{w[0], w[1], w[2], w[3]};
        }
        // a query of one key: its probability is 1 for any score, dS is 0 (not what
        // rounding leaves of it)
        if (hi == 0)
            lse2 = INFINITY;
    }

    // At the start of tile j the loads of tile j + 1 have landed (of those issued, up to tile
    // j + BUFS - 2, later ones may be in flight) and every wavefront has finished tile j - 1,
    // so its buffer takes tile j + BUFS - 1.
    static_assert(BUFS == 3 || BUFS == 4, "");
    Cooked y, rest;
    int r0 = 0, cbuf = 0;  // this block's first row, this tile's buffer
    auto begin = [&](int j) {
        if (BUFS == 4 && j + 2 < j1)
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(LOADS));
        else
            __builtin_amdgcn_s_waitcnt(dma_vmcnt(0));
        asm volatile("" ::: "memory");
        __syncthreads();
        if (j + BUFS - 1 < j1)
            fetch();
    };
    auto block = [&](auto subc, const Raw &cur, Raw &nxt) {
        constexpr bool WITHIN = decltype(subc)::value + 1 < SUB;
        const int nbuf = WITHIN ? cbuf : following(cbuf);
        // (the last tile of a head: the next one's first follows)
        const int next = !WITHIN && KEYS && r0 + 32 >= Q.len ? first * BT : r0 + 32;
        if (BIAS)
            bias(next, nxt);
        if (BIAS || (r0 >= free_lo && r0 + 31 <= free_hi))
            run(Flag<false>{}, subc, lds + cbuf, lds + nbuf, r0, cur, nxt, y, rest);
        else
            run(Flag<true>{}, subc, lds + cbuf, lds + nbuf, r0, cur, nxt, y, rest);
        cbuf = nbuf;
        r0 = next;
    };
    auto last = [&](const Raw &cur) {
        const int at = r0 + 4 * hf;
        each<PAIRS>([&](auto ic) {
            cook(Flag<!BIAS>{}, Flag<TWO>{}, ic, lo - at, hi - at, cur, y, rest);
        });
        second_products(Flag<TWO>{}, Index<SUB - 1>{}, lds + cbuf, y, rest);
    };
    if (few) {
        for (int j = j0; j < j1; ++j) {
            if (KEYS && j > j0 && (j - j0) % BUFS == 0) {
                __syncthreads();
                for (int i = j; i < min(j1, j + BUFS); ++i)
                    fetch();
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
            }
            each<SUB>([&](auto subc) {
                const uint8_t *const buf = lds + (j - l0) % BUFS * BUF;
                const int at = (first + (KEYS ? j % tiles : j)) * BT + 32 * decltype(subc)::value;
                const int from = lo - at - 4 * hf, to = hi - at - 4 * hf;
                Raw x;
                first_products(subc, buf, at, x);
                each<PAIRS>([&](auto ic) {
                    cook(Flag<true>{}, Flag<true>{}, ic, from, to, x, y, rest);
                });
                second_products(Flag<false>{}, subc, buf, y, y);
                second_products(Flag<false>{}, subc, buf, rest, rest);
            });
        }
    } else if (j0 < j1) {
        Raw xa, xb;
        r0 = (first + (KEYS ? j0 % tiles : j0)) * BT;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        first_products(Index<0>{}, lds, r0, xa);
        int j = j0;
        if constexpr (SUB == 2) {
            for (; j + 1 < j1; ++j) {
                begin(j);
                block(Index<0>{}, xa, xb);
                block(Index<1>{}, xb, xa);
            }
            block(Index<0>{}, xa, xb);
            last(xb);
        } else {
            for (; j + 2 < j1; j += 2) {
                begin(j);
                block(Index<0>{}, xa, xb);
                begin(j + 1);
                block(Index<0>{}, xb, xa);
            }
            if (j + 1 < j1) {
                begin(j);
                block(Index<0>{}, xa, xb);
                last(xb);
            } else {
                last(xa);
            }
        }
    }

    // channel 32 d + 8 e + 4 hf + r % 4 of the lane's row; padding rows: zeros
    if (t >= (KEYS ? K.cap : Q.cap))
        return;
    auto store = [&](const f32x16 (&acc)[DT], void *out, int64_t ld, float *to, float f) {
        const int64_t at = ((KEYS ? K.first : Q.first) + t) * ld + head * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int ch = 32 * d + 8 * e + 4 * hf;
                f32x4_t v;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = live ? acc[d][4 * e + i] * f : 0.0f;
                if (parts > 1)
                    *reinterpret_cast<f32x4_t *>(
                        to + (((int64_t)part * s.B * s.Hk + unit) * rows + row) * D + ch) = v;
                else if (a.bf16)
                    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(out) + at + ch) =
                        u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                else
                    *reinterpret_cast<f32x4_t *>(static_cast<float *>(out) + at + ch) = v;
            }
    };
    if constexpr (KEYS) {
        // (of a single key: dS is 0, as for its queries)
        store(acc1, a.dk, a.lddk, a.part, K.len == 1 ? 0.0f : a.scale);
        store(acc2, a.dv, a.lddv, a.part + (int64_t)parts * s.B * s.Hk * rows * D, 1.0f);
    } else {
        store(acc1, a.dq, a.lddq, a.part, a.scale);
    }
}

// Partial sums added in order, 4 channels a thread (blockIdx.y: dk, dv).  4 parts of 16384
// rows of 128 for both: 12 us, 6.2 TB/s, much of it from the last-level cache.
template <int D, bool KEYS>
__global__ __launch_bounds__(256) void attn_grad_join_kernel(const SeqAttnGrad a)
{
    const SeqAttn &s = a.s;
    const int G = s.H / s.Hk, parts = KEYS ? a.kparts : a.qparts;
    const int rows = KEYS ? s.KT : s.T * G;
    const int64_t all = (int64_t)s.B * s.Hk * rows, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t at = i / (D / 4);
    const int ch = 4 * (int)(i % (D / 4));
    if (at >= all)
        return;
    const int unit = (int)(at / rows), row = (int)(at - (int64_t)unit * rows);
    const int hk = unit / s.B, b = unit - hk * s.B;
    const int t = KEYS ? row : row / G, head = KEYS ? hk : hk * G + row - t * G;
    const SeqRows R = KEYS ? seq_rows(s.k_off, s.k_len, s.krows, s.KT, b)
                           : seq_rows(s.q_off, s.q_len, s.qrows, s.T, b);
    if (t >= R.cap)
        return;
    const float *const part = a.part + (int64_t)blockIdx.y * parts * all * D + at * D + ch;
    f32x4_t v = *reinterpret_cast<const f32x4_t *>(part);
#pragma unroll 4
    for (int p = 1; p < parts; ++p)
        v += *reinterpret_cast<const f32x4_t *>(part + p * all * D);
    void *const out = !KEYS ? a.dq : blockIdx.y ? a.dv : a.dk;
    const int64_t ld = !KEYS ? a.lddq : blockIdx.y ? a.lddv : a.lddk;
    const int64_t o = (R.first + t) * ld + head * D + ch;
    if (a.bf16)
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(out) + o) =
            u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(out) + o) = v;
}

// Rows of a streamed tile: 64, half the barriers and waits of 32, where the LDS holds them
// (two workgroups on a CU but for D = 128 and kept keys).  Registers: 220 and 230 (dq, dk and
// dv) of 256 for D = 64; for D = 128 dq takes all 256, with 14 values spilled outside of the
// loop over tiles, and kept keys 361 of the 512 that a workgroup alone on its CU has.
constexpr int tile_rows(int D, bool keys) { return D == 64 || keys ? 64 : 32; }
constexpr int on_a_cu(int D, bool keys, bool two) { return D == 64 || !(keys || two) ? 2 : 1; }

int64_t kept(const SeqAttn &s, bool keys)
{
    return keys ? s.KT : (int64_t)s.T * (s.H / s.Hk);
}

bool few_out(const SeqAttn &s, bool keys)
{
    return kept(s, keys) * s.B * s.Hk <= FEW_OUT;
}

int64_t blocks(const SeqAttn &s, bool keys)
{
    return (kept(s, keys) + KEEP - 1) / KEEP * s.B * s.Hk;
}

// us of a launch (fitted to sweeps of 247 shapes in up to 8 numbers of parts; the choice
// takes 1.01 times the best one's time on average, 1.07 at the ninth decile): its start
// and end, a block of 32 streamed rows where a workgroup has its CU to itself, and where two
// share it; by D = 64 and 128 of kept queries, then of kept keys.
struct StepCost {
    double start, alone, shared;
};
constexpr StepCost STEP[2][2] = {{{6.95, 0.41, 0.95}, {10.45, 0.73, 1.61}},
                                 {{5.21, 0.64, 0.64}, {7.72, 0.97, 0.97}}};
constexpr double JOIN_US = 2.0, JOIN_PART_US = 0.09;  // of adding parts up, and a part more
constexpr double JOIN_RATE = 4.3e6;                   // bytes a us of their values

double parts_us(const SeqAttn &s, bool keys, int parts)
{
    const StepCost &c = STEP[keys][s.dh == 128];
    const bool two = on_a_cu(s.dh, keys, few_out(s, keys)) == 2;
    const int G = s.H / s.Hk;
    const double w = (double)blocks(s, keys) * parts, slots = (two ? 2.0 : 1.0) * s.cus;
    const double most = std::ceil((keys ? s.T : s.KT) / 32.0) * (keys ? G : 1);
    const double mean = s.causal ? most / 2 + 2 * (keys ? G : 1) : most;
    const double full = std::min(1.0, std::max(0.0, (w - s.cus) / s.cus));
    const double step = two ? c.alone + (c.shared - c.alone) * full : c.alone;
    auto steps = [&](double n) { return std::ceil(n / parts); };
    double us = c.start + (s.causal ? std::max(steps(most) * c.alone,
                                               steps(mean) * step * std::max(1.0, w / slots))
                                    : steps(most) * step * std::ceil(w / slots));
    if (parts > 1) {
        const double rows = (keys ? 2.0 * s.KT : (double)s.T * G) * s.B * s.Hk;
        us += JOIN_US + JOIN_PART_US * parts + parts * rows * s.dh * 8.0 / JOIN_RATE;
    }
    return us;
}

template <int D, bool KEYS>
hipError_t go(const SeqAttnGrad &g, hipStream_t stream)
{
    SeqAttnGrad a = g;
    const int parts = KEYS ? a.kparts : a.qparts;
    const unsigned grid = (unsigned)(blocks(a.s, KEYS) * parts);
    const bool two = few_out(a.s, KEYS);
    if (grid)
        order_work(a.s, grid / ((int64_t)a.s.B * a.s.Hk), on_a_cu(D, KEYS, two));
    constexpr int BT = tile_rows(D, KEYS), BUFS = BT == 64 ? 3 : 4;
    if (grid && two)
        hipLaunchKernelGGL((seq_attn_grad_kernel<D, KEYS, BT, BUFS, true>), dim3(grid),
                           dim3(THREADS), 0, stream, a);
    else if (grid)
        hipLaunchKernelGGL((seq_attn_grad_kernel<D, KEYS, BT, BUFS, false>), dim3(grid),
                           dim3(THREADS), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts < 2 || !grid)
        return e;
    const int64_t threads = (int64_t)a.s.B * a.s.Hk * kept(a.s, KEYS) * (D / 4);
    hipLaunchKernelGGL((attn_grad_join_kernel<D, KEYS>),
                       dim3((unsigned)((threads + 255) / 256), KEYS ? 2 : 1), dim3(256), 0, stream,
                       a);
    return hipGetLastError();
}

}  // namespace

// The number of parts estimated to be fastest.  Measured, us of dk and dv in 1 / 2 / 4 / 8 parts:
// 250 keys of one head of 128 for 4 causal query heads 41.9 / 27.6 / 19.5 / 15.9; 432 keys, 3
// sequences of 4 such 59.7 / 42.0 / 31.4 / 40.6; 778 causal keys, 3 of 8 of 64, one query head
// each 21.5 / 31.1 / 30.6 / 38.6.
SeqAttnGradPlan seq_attn_grad_plan(const SeqAttn &s, bool keys)
{
    constexpr int PARTS[] = {1, 2, 3, 4, 6, 8, 12, 16};
    constexpr int64_t MOST = 1024;  // workgroups of a launch in parts: they bound the workspace
    auto choose = [&](bool k) {
        const int64_t w = blocks(s, k);
        const int64_t tiles =
            k ? ((int64_t)s.T + 63) / 64 * (s.H / s.Hk) : ((int64_t)s.KT + 63) / 64;
        int best = 1;
        double us = 0.0;
        for (const int p : PARTS) {
            if (p > 1 && (p > tiles || w * p > MOST))
                break;
            const double t = parts_us(s, k, p);
            if (p == 1 || t < us) {
                us = t;
                best = p;
            }
        }
        return best;
    };
    return {choose(false), keys ? choose(true) : 1};
}

int64_t seq_attn_grad_workgroups(const SeqAttn &s, const SeqAttnGradPlan &p)
{
    const int64_t q = blocks(s, false) * p.qparts, k = blocks(s, true) * p.kparts;
    return q > k ? q : k;
}

size_t seq_attn_grad_bytes(const SeqAttn &s, const SeqAttnGradPlan &p)
{
    const size_t sums = (size_t)16 * s.H * s.qrows;
    size_t q = 0, k = 0;
    if (p.qparts > 1)
        q = (size_t)p.qparts * s.B * s.H * s.T * s.dh * 4;
    if (p.kparts > 1)
        k = (size_t)2 * p.kparts * s.B * s.Hk * s.KT * s.dh * 4;
    return sums + (q > k ? q : k);
}

hipError_t launch_seq_attn_grad(const SeqAttnGrad &g, hipStream_t stream)
{
    SeqAttnGrad a = g;
    a.part = a.sums + (size_t)4 * a.s.H * a.s.qrows;
    const hipError_t e = a.s.dh == 64 ? go<64, false>(a, stream) : go<128, false>(a, stream);
    if (e != hipSuccess || !a.dk)
        return e;
    return a.s.dh == 64 ? go<64, true>(a, stream) : go<128, true>(a, stream);
}

}  // namespace qlk
