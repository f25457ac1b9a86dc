// Masked attention: sequences of unlike lengths, causal masks, query heads that share
// key heads, few queries over long caches, and the logarithms of the row sums that the
// backward pass starts from.  For query i of a head with n queries and m keys
//
//   O_i = sum_j p_ij V_j / l_i,  p_ij = exp(s_ij - max),  s_ij = scale <Q_i, K_j>,
//   l_i = sum_j p_ij,  lse_i = max + log l_i,  j < m, and with causal j <= i + m - n
//
// in one pass over the keys with a running maximum and sum (online softmax).  The
// products and their layout are those of attention.hip: S^T = K Q^T (a lane holds
// scores of one query), then O^T += V^T P^T with P^T straight from the score
// registers; a lane's query never changes, so its maximum, sum, mask and rescaling
// are its own.  Tiles of keys come in by direct-to-LDS loads, two buffers each for K
// and V, one tile apart.  Matrix and vector units run beside each other within a
// wavefront: the softmax of tile j is placed, a few instructions at a time, between the
// matrix instructions that form the scores of tile j + 1 and the value product of tile
// j - 1.  (In the compiler's order one unit waits for the other: 200 us for 183 of the first
// case below, 118 for 62 of the causal one with 128 channels.)
//
// Rows of a tile are (query, head of the group) pairs, i = t G + g for the G query
// heads of a key head: each K and V tile is read once for all of them, and one token's
// G heads fill G rows.  KG groups of wavefronts share out a tile's keys (KG = 4: one
// wavefront of 32 rows each, for one token; merged through LDS at the end); beyond that
// `splits` workgroups take parts of the keys and attn_join_kernel adds them up.
//
// What bounds it, measured in us: 4096 queries and keys of 32 heads of 64 170 to 180, 760
// to 810 TFLOP/s, by the vector instructions that a score takes (they are active in 0.65 of
// a CU's cycles, the matrix cores in 0.40; LDS in 0.20, without conflicts); of 16 heads of
// 128, twice the matrix work for a score, 149, 920 TFLOP/s.  2 causal sequences of 4096, 32
// heads of 64: 180.  One causal sequence of 2048, 8 key heads of 128 with 4 query heads
// each: 60 to 63, where half of the time without a mask is 42: a grid that the GPU holds at
// once, so the start and end of a launch and what its CUs' last blocks leave idle (two groups
// of wavefronts take as long; two parts of the keys 59 and 17 for the join).  One token of 8
// sequences over up to 8192 keys: 47, 4.4 TB/s, by HBM.
//
// Two workgroups a CU, 256 registers a lane, all of them taken (10 values spilled for D = 64,
// 7 and 3 for D = 128 in one and two groups, outside of the loop over tiles): with three
// workgroups the compiler spills within it (D = 64, tiles of 32 keys: 350 us for 170).  Tiles
// of 64 keys for D = 64; 32 for D = 128 (64, with one workgroup a CU: 68 for 60).  Plain
// stores: non-temporal ones took as long.
#include <algorithm>
#include <cmath>

#include "attn.h"

namespace qlk {
namespace {

constexpr int THREADS = 256;
// The running maximum may trail the true one by 2^LAZY in the exponent (as in
// attention.hip): the quotient O / l is the same for any.
constexpr float LAZY = 8.0f;
constexpr float LN2 = 0.693147180559945309f;

template <int D, int KG, int BK>
__global__ __launch_bounds__(THREADS)
__attribute__((amdgpu_waves_per_eu(D == 128 && KG == 4 ? 1 : 2, 2)))
void seq_attn_kernel(const SeqAttnOut a)
{
    constexpr int GT = THREADS / KG, GW = GT / 64;  // threads, wavefronts of a key group
    constexpr int BQ = 32 * GW;                     // rows of the workgroup
    constexpr int TILE = BK * D * 2;                // bytes
    constexpr int SUB = BK / 32, DT = D / 32, DS = D / 16;
    __shared__ __align__(16) uint8_t lds[KG * 4 * TILE];
    const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / GT);
    const int tid = (int)threadIdx.x - kg * GT, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hf = lane >> 5;
    uint8_t *const mine = lds + kg * 4 * TILE;
    auto kbuf = [&](int i) { return mine + i * TILE; };
    auto vbuf = [&](int i) { return mine + (2 + i) * TILE; };

    const SeqAttn &s = a.s;
    const int G = s.H / s.Hk;
    const int nq = (s.T * G + BQ - 1) / BQ;
    const Work w = work_of(s, (int)blockIdx.x, (int)gridDim.x, a.splits, nq);
    const int part = w.part, unit = w.unit, hk = unit / s.B, b = unit - hk * s.B;
    const int qblk = s.causal ? nq - 1 - w.blk : w.blk;
    const SeqRows Q = seq_rows(s.q_off, s.q_len, s.qrows, s.T, b);
    const SeqRows K = seq_rows(s.k_off, s.k_len, s.krows, s.KT, b);
    const int row0 = qblk * BQ;
    if (row0 >= Q.cap * G)
        return;
    const int row = row0 + wave * 32 + l32, t = row / G, g = row - t * G;
    const int head = hk * G + g;
    const bool live = t < Q.len;

    // the last key of this lane's query, of any query of the workgroup, and of the
    // wavefront's first: tiles up to that one need no mask
    auto last_of = [&](int q) {
        return s.causal ? min(K.len - 1, q + K.len - Q.len) : K.len - 1;
    };
    const int tmax = min((row0 + BQ - 1) / G, Q.len - 1);
    const int keys = Q.len > row0 / G ? max(0, last_of(tmax) + 1) : 0;
    const int tiles = (keys + BK - 1) / BK;
    const int kt0 = (int)((int64_t)tiles * part / a.splits);
    const int kt1 = (int)((int64_t)tiles * (part + 1) / a.splits);
    const int lim = live ? min(last_of(t), kt1 * BK - 1) : -1;
    const int free_keys = last_of((row0 + wave * 32) / G) + 1;

    bf16x8 qb[DS];
#pragma unroll
    for (int i = 0; i < DS; ++i) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if (live)
            v = *reinterpret_cast<const u32x4 *>(s.q + (Q.first + t) * s.ldq + head * D + 16 * i +
                                                 8 * hf);
        qb[i] = __builtin_bit_cast(bf16x8, v);
    }

    const uint8_t *const kbase =
        reinterpret_cast<const uint8_t *>(s.k + K.first * s.ldk + hk * D);
    const uint8_t *const vbase =
        reinterpret_cast<const uint8_t *>(s.v + K.first * s.ldv + hk * D);
    TileLoad<D, BK, GT> kload, vload;
    kload.init(s.ldk, tid);
    vload.init(s.ldv, tid);
    // K and V of this group's next tiles (counted on: scalar instructions take their turn
    // with the others of a wavefront).  This group's tiles: kt0 + KG j + kg, j < n; one past
    // kt1 is loaded as the last tile again (every key of it lies past lim).
    const int n = (kt1 - kt0 + KG - 1) / KG;
    auto tile_at = [&](int j) { return kt0 + KG * j + kg; };
    struct Next {
        const uint8_t *p;
        int left;
    } nextk, nextv;
    {
        const int kt = max(0, min(kt0 + kg, kt1 - 1));
        nextk = {kbase + (int64_t)kt * BK * s.ldk * 2, K.len - kt * BK};
        nextv = {vbase + (int64_t)kt * BK * s.ldv * 2, K.len - kt * BK};
    }
    // (keys from the next tile's first to kt1's: no more than those of the tile itself)
    const int beyond = K.len - kt1 * BK;
    auto fetch = [&](const TileLoad<D, BK, GT> &load, Next &x, int64_t ld, uint8_t *buf) {
        load.issue(x.p, x.left, ld, buf, tid);
        const int tiles_on = KG == 1 || x.left - beyond > KG * BK
                                 ? KG
                                 : (x.left - beyond + BK - 1) / BK - 1;
        x.p += tiles_on * (BK * 2 * ld);
        x.left -= tiles_on * BK;
    };
    auto fetch_k = [&](uint8_t *buf) { fetch(kload, nextk, s.ldk, buf); };
    auto fetch_v = [&](uint8_t *buf) { fetch(vload, nextv, s.ldv, buf); };

    f32x16 oacc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            oacc[d][r] = 0.0f;
    float mrun = -INFINITY, lrun = 0.0f;
    const float c = s.c;
    // Softmax of a tile's scores in PARTS parts, to be placed between matrix instructions:
    // its maximum, the factor that brings the sums so far to it, then the probabilities as
    // operands, two at a time.  Score r of subtile sub is key kt BK + 32 sub + 8 (r / 4) + 4
    // hf + r % 4.
    // D = 128 (one code for every tile, or the registers run out): the mask is what a
    // tile's scores start from, 0 or -infinity.
    constexpr bool BIAS = D == 128;
    constexpr int MAXES = 4 * SUB, PAIRS = 8 * SUB, PARTS = MAXES + 1 + PAIRS;
    float mx[2], ls[2], mc, alpha;
    auto softmax = [&](auto maskc, auto ic, int left, const f32x16 (&sc)[SUB],
                       bf16x8 (&pb)[SUB][2]) {
        constexpr bool MASK = decltype(maskc)::value;
        constexpr int I = decltype(ic)::value;
        auto in = [&](int sub, int r) { return 32 * sub + 8 * (r >> 2) + (r & 3) <= left; };
        if constexpr (I < MAXES) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int sub = I / 4, r = 4 * (I % 4) + e;
                const float x = !MASK || in(sub, r) ? sc[sub][r] : -INFINITY;
                mx[e & 1] = I == 0 && e < 2 ? x : fmaxf(mx[e & 1], x);
            }
        } else if constexpr (I == MAXES) {
            float lo, hi;
            both_halves(fmaxf(mx[0], mx[1]), lo, hi);
            const float mt = fmaxf(lo, hi);
            // the maximum moves only where the scores exceed it by more than LAZY (no score
            // at all: it stays at -inf; c > 0, so that the factor from there is 0)
            const bool up = mt > mrun && !((mt - mrun) * c <= LAZY);
            const float mnew = up ? mt : mrun;
            alpha = up ? __builtin_amdgcn_exp2f((mrun - mnew) * c) : 1.0f;
            mrun = mnew;
            mc = BIAS && mrun == -INFINITY ? 0.0f : mrun * c;
        } else {
            constexpr int p = I - MAXES - 1, sub = p / 8, r = 2 * (p % 8);
            float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[sub][r], c, -mc));
            float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[sub][r + 1], c, -mc));
            if (MASK) {
                p0 = in(sub, r) ? p0 : 0.0f;
                p1 = in(sub, r + 1) ? p1 : 0.0f;
            }
            ls[0] = p == 0 ? p0 : ls[0] + p0;
            ls[1] = p == 0 ? p1 : ls[1] + p1;
            u32x4 w = __builtin_bit_cast(u32x4, pb[sub][r / 8]);
            w[r / 2 % 4] = pack_bf16(p0, p1);
            pb[sub][r / 8] = __builtin_bit_cast(bf16x8, w);
            if constexpr (I == PARTS - 1)
                lrun = __builtin_fmaf(lrun, alpha, ls[0] + ls[1]);
        }
    };
    auto rescale = [&] {
        if (__ballot(alpha != 1.0f) != 0) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    oacc[d][r] *= alpha;
        }
    };
    auto bias = [&](int kt, f32x16 (&sc)[SUB]) {
        const int left = lim - kt * BK - 4 * hf;
        if (BIAS && kt < kt1 && (kt + 1) * BK <= free_keys) {
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sc[sub][r] = 0.0f;
        } else if (BIAS) {
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sc[sub][r] = 32 * sub + 8 * (r >> 2) + (r & 3) <= left ? 0.0f : -INFINITY;
        }
    };
    // The matrix instructions of a step, one by one: the scores of a tile (K in ks), then
    // the value product with the probabilities pb (V in vt).
    constexpr int SCORES = SUB * DS, PRODUCTS = 2 * SUB * DT;
    auto operand = [&](auto ic, const uint8_t *ks, const uint8_t *vt) {
        constexpr int I = decltype(ic)::value;
        if constexpr (I < SCORES)
            return row_operand<D>(ks, 32 * (I % SUB) + l32, I / SUB, hf);
        else
            return transposed_operand<D>(vt, (I - SCORES) / DT, (I - SCORES) % DT, lane);
    };
    auto multiply = [&](auto ic, bf16x8 w, f32x16 (&sc)[SUB], const bf16x8 (&pb)[SUB][2]) {
        constexpr int I = decltype(ic)::value;
        if constexpr (I < SCORES) {
            constexpr int sub = I % SUB, i = I / SUB;
            const f32x16 zero = {};
            sc[sub] = mfma(w, qb[i], i == 0 && !BIAS ? zero : sc[sub]);
        } else {
            constexpr int kc = (I - SCORES) / DT, d = (I - SCORES) % DT;
            oacc[d] = mfma(w, pb[kc / 2][kc % 2], oacc[d]);
        }
    };
    // Matrix instructions FROM .. TO - 1 with the parts of a softmax spread between them,
    // operands read AHEAD of them.
    constexpr int AHEAD = 3;
    auto run = [&](auto fromc, auto toc, auto maskc, int kt, const f32x16 (&cur)[SUB],
                   f32x16 (&nxt)[SUB], const bf16x8 (&pold)[SUB][2], bf16x8 (&pnew)[SUB][2],
                   const uint8_t *ks, const uint8_t *vt) {
        constexpr int FROM = decltype(fromc)::value, N = decltype(toc)::value - FROM;
        const int left = lim - kt * BK - 4 * hf;
        bf16x8 w[AHEAD + 1];
        each<AHEAD>([&](auto ic) {
            constexpr int I = decltype(ic)::value;
            if constexpr (I < N)
                w[I] = operand(Index<FROM + I>{}, ks, vt);
        });
        each<N>([&](auto ic) {
            constexpr int I = decltype(ic)::value;
            if constexpr (I + AHEAD < N)
                w[(I + AHEAD) % (AHEAD + 1)] = operand(Index<FROM + I + AHEAD>{}, ks, vt);
            multiply(Index<FROM + I>{}, w[I % (AHEAD + 1)], nxt, pold);
            constexpr int P0 = PARTS * I / N, P1 = PARTS * (I + 1) / N;
            each<P1 - P0>([&](auto pc) {
                softmax(maskc, Index<P0 + decltype(pc)::value>{}, left, cur, pnew);
            });
            keep_order();
        });
    };
    auto scores = [&](const uint8_t *ks, f32x16 (&sc)[SUB]) {
        const bf16x8 none[SUB][2] = {};
        each<SCORES>([&](auto ic) { multiply(ic, operand(ic, ks, ks), sc, none); });
    };
    auto product = [&](const uint8_t *vt, const bf16x8 (&pb)[SUB][2]) {
        f32x16 none[SUB];
        each<PRODUCTS>([&](auto ic) {
            constexpr int I = SCORES + decltype(ic)::value;
            multiply(Index<I>{}, operand(Index<I>{}, vt, vt), none, pb);
        });
    };

    // Step j: the softmax of tile j on the vector units, and beside it, independent of it,
    // the scores of tile j + 1 and the value product of tile j - 1 on the matrix cores.  At
    // its start every load issued so far has landed (K of tile j + 1, V of tile j - 1)
    // and every wavefront has finished the step before it: K's buffer of tile j takes tile
    // j + 2, V's of tile j - 2 takes tile j.
    auto step = [&](auto oddc, auto maskc, int j, const f32x16 (&cur)[SUB], f32x16 (&nxt)[SUB],
                    const bf16x8 (&pold)[SUB][2], bf16x8 (&pnew)[SUB][2]) {
        constexpr int P = decltype(oddc)::value ? 1 : 0;
        bias(tile_at(j + 1), nxt);
        run(Index<0>{}, Index<SCORES + PRODUCTS>{}, maskc, tile_at(j), cur, nxt, pold, pnew,
            kbuf(P ^ 1), vbuf(P ^ 1));
        rescale();
    };
    auto begin = [&](auto oddc, int j) {
        constexpr int P = decltype(oddc)::value ? 1 : 0;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (j + 2 < n)
            fetch_k(kbuf(P));
        fetch_v(vbuf(P));
    };
    auto middle = [&](auto oddc, int j, const f32x16 (&cur)[SUB], f32x16 (&nxt)[SUB],
                      const bf16x8 (&pold)[SUB][2], bf16x8 (&pnew)[SUB][2]) {
        begin(oddc, j);
        const int kt = tile_at(j);
        if (!BIAS && (kt >= kt1 || (kt + 1) * BK > free_keys))
            step(oddc, Flag<true>{}, j, cur, nxt, pold, pnew);
        else
            step(oddc, Flag<false>{}, j, cur, nxt, pold, pnew);
    };
    auto last = [&](auto oddc, int j, const f32x16 (&cur)[SUB], const bf16x8 (&pold)[SUB][2],
                    bf16x8 (&pnew)[SUB][2]) {
        constexpr int P = decltype(oddc)::value ? 1 : 0;
        f32x16 none[SUB];
        begin(oddc, j);
        run(Index<SCORES>{}, Index<SCORES + PRODUCTS>{}, Flag<!BIAS>{}, tile_at(j), cur, none, pold,
            pnew, vbuf(P ^ 1), vbuf(P ^ 1));
        rescale();
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        product(vbuf(P), pnew);
    };
    if (n > 0) {
        fetch_k(kbuf(0));
        fetch_v(vbuf(0));
        if (n > 1)
            fetch_k(kbuf(1));
        f32x16 sa[SUB], sb[SUB];
        bf16x8 pa[SUB][2], pz[SUB][2];
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        bias(tile_at(0), sa);
        scores(kbuf(0), sa);
        if (n > 1) {
            // step 0: no value product yet
            if (n > 2) {
                __syncthreads();
                fetch_k(kbuf(0));
            }
            bias(tile_at(1), sb);
            run(Index<0>{}, Index<SCORES>{}, Flag<!BIAS>{}, tile_at(0), sa, sb, pz, pa, kbuf(1),
                kbuf(1));
            int j = 1;
            for (; j + 2 < n; j += 2) {
                middle(Flag<true>{}, j, sb, sa, pa, pz);
                middle(Flag<false>{}, j + 1, sa, sb, pz, pa);
            }
            if (j + 1 < n) {
                middle(Flag<true>{}, j, sb, sa, pa, pz);
                last(Flag<false>{}, j + 1, sa, pz, pa);
            } else {
                last(Flag<true>{}, j, sb, pa, pz);
            }
        } else {
            const int left = lim - tile_at(0) * BK - 4 * hf;
            each<PARTS>([&](auto ic) { softmax(Flag<!BIAS>{}, ic, left, sa, pa); });
            product(vbuf(0), pa);
        }
    }
    {
        float lo, hi;
        both_halves(lrun, lo, hi);
        lrun = lo + hi;
    }

    if constexpr (KG > 1) {
        // the other groups' states through LDS (over the buffers, which every wavefront
        // has finished with), [value][lane] per wavefront; group 0 adds them in order
        constexpr int VALUES = 2 + 16 * DT;
        static_assert((KG - 1) * GW * VALUES * 64 * 4 <= KG * 4 * TILE, "");
        __syncthreads();
        if (kg > 0) {
            float *const x =
                reinterpret_cast<float *>(lds) + ((kg - 1) * GW + wave) * VALUES * 64 + lane;
            x[0] = mrun;
            x[64] = lrun;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x[(2 + 16 * d + r) * 64] = oacc[d][r];
        }
        __syncthreads();
        if (kg > 0)
            return;
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const float *const x =
                reinterpret_cast<const float *>(lds) + ((k - 1) * GW + wave) * VALUES * 64 + lane;
            const float m1 = x[0], m = fmaxf(mrun, m1);
            const float a0 = mrun == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mrun - m) * c);
            const float a1 = m1 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m1 - m) * c);
            mrun = m;
            lrun = a0 * lrun + a1 * x[64];
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    oacc[d][r] = a0 * oacc[d][r] + a1 * x[(2 + 16 * d + r) * 64];
        }
    }

    // channel 32 d + 8 e + 4 hf + r % 4 of the lane's row
    if (t >= Q.cap)
        return;
    if (a.splits > 1) {
        const int64_t at = ((int64_t)part * s.B * s.Hk + unit) * s.T * G + row;
        float *const o = a.part + at * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<f32x4_t *>(o + 32 * d + 8 * e + 4 * hf) =
                    f32x4_t{oacc[d][4 * e], oacc[d][4 * e + 1], oacc[d][4 * e + 2],
                            oacc[d][4 * e + 3]};
        if (hf == 0)
            *reinterpret_cast<f32x2_t *>(a.part +
                                         (int64_t)a.splits * s.B * s.Hk * s.T * G * D + at * 2) =
                f32x2_t{mrun, lrun};
        return;
    }
    // no key: zeros (also of a padding row)
    const bool none = lim < 0;
    const float inv = 1.0f / lrun;
    const int64_t orow = (Q.first + t) * a.ldo + head * D;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ch = 32 * d + 8 * e + 4 * hf;
            f32x4_t v;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = none ? 0.0f : oacc[d][4 * e + i] * inv;
            if (a.obf16)
                *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.o) + orow + ch) =
                    u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            else
                *reinterpret_cast<f32x4_t *>(static_cast<float *>(a.o) + orow + ch) = v;
        }
    if (a.lse && hf == 0)
        a.lse[head * s.qrows + Q.first + t] =
            none ? -INFINITY : (mrun * c + __builtin_amdgcn_logf(lrun)) * LN2;
}

// The parts of a split, joined in order: 4 channels of a (query, head) a thread.  (Latency:
// 4 parts of 256 rows of 128 take 4.8 us.)
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(const SeqAttnOut a)
{
    const SeqAttn &s = a.s;
    const int G = s.H / s.Hk;
    const int64_t rows = (int64_t)s.B * s.Hk * s.T * G;
    const int64_t i = (int64_t)blockIdx.x * 256 + (int)threadIdx.x, at = i / (D / 4);
    const int ch = 4 * (int)(i % (D / 4));
    if (at >= rows)
        return;
    const int unit = (int)(at / (s.T * G)), row = (int)(at - (int64_t)unit * s.T * G);
    const int hk = unit / s.B, b = unit - hk * s.B;
    const int t = row / G, head = hk * G + row - t * G;
    const f32x2_t *const ml =
        reinterpret_cast<const f32x2_t *>(a.part + a.splits * rows * D) + at;
    const float *const po = a.part + at * D + ch;
    // as in the kernel, part by part: 0 where a part saw no key
    f32x2_t x = ml[0];
    float m = x[0], l = x[1];
    f32x4_t o = *reinterpret_cast<const f32x4_t *>(po);
#pragma unroll 4
    for (int p = 1; p < a.splits; ++p) {
        x = ml[p * rows];
        const f32x4_t op = *reinterpret_cast<const f32x4_t *>(po + p * rows * D);
        const float mn = fmaxf(m, x[0]);
        const float w0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - mn) * s.c);
        const float w1 = x[0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((x[0] - mn) * s.c);
        m = mn;
        l = w0 * l + w1 * x[1];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            o[k] = w0 * o[k] + w1 * op[k];
    }
    const SeqRows Q = seq_rows(s.q_off, s.q_len, s.qrows, s.T, b);
    if (t >= Q.cap)
        return;
    const SeqRows K = seq_rows(s.k_off, s.k_len, s.krows, s.KT, b);
    const bool none = t >= Q.len || K.len == 0 || (s.causal && t + K.len - Q.len < 0);
    const float inv = 1.0f / l;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        o[k] = none ? 0.0f : o[k] * inv;
    const int64_t out = (Q.first + t) * a.ldo + head * D + ch;
    if (a.obf16)
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.o) + out) =
            u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    else
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(a.o) + out) = o;
    if (a.lse && ch == 0)
        a.lse[head * s.qrows + Q.first + t] =
            none ? -INFINITY : (m * s.c + __builtin_amdgcn_logf(l)) * LN2;
}

int tile_rows(int groups) { return 128 / groups; }
int on_a_cu(const SeqAttn &s, int groups) { return s.dh == 64 || groups < 4 ? 2 : 1; }

// us of a launch (fitted to sweeps of 398 shapes in up to 40 forms each; the choice takes
// 1.015 times the best form's time on average, 1.06 at the ninth decile): its start and end,
// 64 keys of a group of wavefronts where a workgroup has its CU to itself, and where two
// share it.
struct StepCost {
    double start, alone, shared;
};
constexpr StepCost STEP[2][3] = {{{4.81, 0.80, 1.30}, {4.90, 0.87, 1.88}, {4.58, 1.34, 2.58}},
                                 {{5.01, 1.37, 1.57}, {5.33, 1.58, 2.74}, {5.65, 2.22, 2.22}}};
constexpr double JOIN_US = 2.0, JOIN_PART_US = 0.13;  // of joining parts, and a part more
constexpr double JOIN_RATE = 1.9e6, KEY_RATE = 6.5e6;  // bytes a us: their values; keys

double form_us(const SeqAttn &s, int groups, int splits)
{
    const int kind = groups == 4 ? 2 : groups - 1;
    const StepCost &c = STEP[s.dh == 128][kind];
    const bool two = on_a_cu(s, groups) == 2;
    const double units = (double)s.B * s.Hk, rows = (double)s.T * (s.H / s.Hk);
    const double w = std::ceil(rows / tile_rows(groups)) * units * splits;
    const double slots = (two ? 2.0 : 1.0) * s.cus;
    const double most = std::ceil(s.KT / 64.0);
    // (causal: the longest of a launch's chains, and the average that fills its places)
    const double mean =
        s.causal ? std::max(1.0, (s.KT - 0.5 * std::min(s.T, s.KT)) / 64.0 + 0.5) : most;
    auto steps = [&](double tiles) { return std::ceil(tiles / splits / groups); };
    const double full = std::min(1.0, std::max(0.0, (w - s.cus) / s.cus));
    const double step = two ? c.alone + (c.shared - c.alone) * full : c.alone;
    const double rounds = s.causal ? std::max(1.0, w / slots) : std::ceil(w / slots);
    double us = std::max(s.causal ? steps(most) * c.alone : 0.0, steps(mean) * step * rounds);
    // (of two bounds near each other both count)
    const double bytes_us = units * s.KT * s.dh * 4.0 / KEY_RATE;
    const double a2 = us * us, b2 = bytes_us * bytes_us;
    us = c.start + std::sqrt(std::sqrt(a2 * a2 + b2 * b2));
    if (splits > 1)
        us += JOIN_US + JOIN_PART_US * splits +
              splits * units * rows * (s.dh + 2) * 4.0 / JOIN_RATE;
    return us;
}

}  // namespace

// The form estimated to be fastest.  Measured, us in 1, 2 and 4 groups of unsplit and of
// the best number of parts (queries x keys, heads): 1 x 5066, 8 sequences of 16 of 64 65.5 /
// 43.7 / 41.4 and 34.9 / 32.2 / 31.2 (4 parts); 592 x 592, 3 of 8 of 64, causal 13.0 / 9.7 / -;
// 215 x 215, 3 of 8 of 128, 4 query heads each 12.3 / 13.1 / -, in 2 parts 26.3 / 28.5 / -.
SeqAttnPlan seq_attn_plan(const SeqAttn &s)
{
    // (96: as far as the sweeps went; one sequence with one key head stays below the CUs)
    constexpr int SPLITS[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96};
    constexpr int64_t MOST = 1024;  // workgroups of a split launch: they bound the workspace
    const int64_t rows = (int64_t)s.T * (s.H / s.Hk), tiles = ((int64_t)s.KT + 63) / 64;
    SeqAttnPlan best{1, 1};
    double us = 0.0;
    for (int groups = 1; groups <= (rows <= 128 ? 4 : 2); groups *= 2)
        for (const int splits : SPLITS) {
            const SeqAttnPlan p{groups, splits};
            if (splits > 1 && (splits > tiles || seq_attn_workgroups(s, p) > MOST))
                break;
            const double t = form_us(s, groups, splits);
            if ((groups == 1 && splits == 1) || t < us) {
                us = t;
                best = p;
            }
        }
    return best;
}

int64_t seq_attn_workgroups(const SeqAttn &s, const SeqAttnPlan &p)
{
    const int64_t rows = (int64_t)s.T * (s.H / s.Hk);
    return (rows + tile_rows(p.groups) - 1) / tile_rows(p.groups) * s.B * s.Hk * p.splits;
}

size_t seq_attn_bytes(const SeqAttn &s, const SeqAttnPlan &p)
{
    return p.splits < 2 ? 0 : (size_t)p.splits * s.B * s.H * s.T * (s.dh + 2) * 4;
}

hipError_t launch_seq_attn(const SeqAttnOut &out, const SeqAttnPlan &p, hipStream_t stream)
{
    SeqAttnOut a = out;
    const int64_t workgroups = seq_attn_workgroups(a.s, p);
    order_work(a.s, workgroups / ((int64_t)a.s.B * a.s.Hk), on_a_cu(a.s, p.groups));
    const dim3 grid((unsigned)workgroups), block(THREADS);
#define QL_GO(D, KG, BK) \
    hipLaunchKernelGGL((seq_attn_kernel<D, KG, BK>), grid, block, 0, stream, a)
    if (a.s.dh == 64) {
        if (p.groups == 1)
            QL_GO(64, 1, 64);
        else if (p.groups == 2)
            QL_GO(64, 2, 64);
        else
            QL_GO(64, 4, 32);
    } else {
        if (p.groups == 1)
            QL_GO(128, 1, 32);
        else if (p.groups == 2)
            QL_GO(128, 2, 32);
        else
            QL_GO(128, 4, 32);
    }
#undef QL_GO
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits < 2)
        return e;
    const dim3 joins((unsigned)(((int64_t)a.s.B * a.s.H * a.s.T * (a.s.dh / 4) + 255) / 256));
    if (a.s.dh == 64)
        hipLaunchKernelGGL(attn_join_kernel<64>, joins, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(attn_join_kernel<128>, joins, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace qlk
