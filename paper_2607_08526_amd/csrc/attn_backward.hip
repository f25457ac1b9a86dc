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
// A wavefront keeps NS x 32 rows of two tensors in registers as right operands (Q, dO; or
// K, V); tiles of BT rows of the other two (K, V; or Q, dO) come into LDS by direct loads,
// two buffers.  For 32 of them at a time, S and dP are formed with the streamed rows as
// left operand: a lane then holds 16 streamed rows of one kept row, just what the right
// operand of the second products (transposed left operand: dQ^T += K^T dS^T, dV^T += dO^T
// P, dK^T += Q^T dS) wants of P and dS, which are rounded to bf16 for it.
#include "attn.h"

namespace qlk {
namespace {

constexpr int THREADS = 256;
constexpr float LOG2E = 1.44269504088896340736f;

// kept rows of a workgroup
template <int NS>
constexpr int KEEP = 128 * NS;

template <int D, bool KEYS, int NS, int BT>
__global__ __launch_bounds__(THREADS)
void seq_attn_grad_kernel(const SeqAttnGrad a)
{
    constexpr int TILE = BT * D * 2;  // bytes of a tile
    constexpr int SUB = BT / 32, DT = D / 32, DS = D / 16;
    constexpr int BUF = 2 * TILE + (KEYS ? 512 : 0);  // (two arrays of 64 sums)
    __shared__ __align__(16) uint8_t lds[2 * BUF];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hf = lane >> 5;

    const SeqAttn &s = a.s;
    const int G = s.H / s.Hk, parts = KEYS ? a.kparts : a.qparts;
    const int rows = KEYS ? s.KT : s.T * G;  // kept, of a (sequence, key head)
    const int nb = (rows + KEEP<NS> - 1) / KEEP<NS>;
    int L = xcd_order((int)blockIdx.x, (int)gridDim.x);
    const int part = L % parts;
    L /= parts;
    const int unit = L / nb, b = unit / s.Hk, hk = unit - b * s.Hk;
    // causal: the longest first (the last queries, the first keys)
    const int blk = s.causal && !KEYS ? nb - 1 - (L - unit * nb) : L - unit * nb;
    const SeqRows Q = seq_rows(s.q_off, s.q_len, s.qrows, s.T, b);
    const SeqRows K = seq_rows(s.k_off, s.k_len, s.krows, s.KT, b);
    const int row0 = blk * KEEP<NS>;
    if (row0 >= (KEYS ? K.cap : Q.cap * G))
        return;
    const int shift = K.len - Q.len;  // causal: query t sees the keys up to t + shift
    const float c = s.c;

    // the kept rows of this lane: a row's operands, and the streamed rows lo to hi that
    // meet it; of the wavefront: the streamed rows that meet all its live rows
    bf16x8 x1[NS][DS], x2[NS][DS];
    int lo[NS], hi[NS];
    float lse2[NS], delta[NS];  // of a kept query
    const int wrow = row0 + wave * 32 * NS;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        const int row = wrow + 32 * n + l32;
        const int t = KEYS ? row : row / G, head = KEYS ? hk : hk * G + row - t * G;
        const bool live = t < (KEYS ? K.len : Q.len);
        const uint16_t *p1 = KEYS ? s.k + (K.first + t) * s.ldk : s.q + (Q.first + t) * s.ldq;
        const uint16_t *p2 = KEYS ? s.v + (K.first + t) * s.ldv : a.dO + (Q.first + t) * a.lddo;
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            u32x4 v1 = {0u, 0u, 0u, 0u}, v2 = v1;
            if (live) {
                v1 = *reinterpret_cast<const u32x4 *>(p1 + head * D + 16 * i + 8 * hf);
                v2 = *reinterpret_cast<const u32x4 *>(p2 + head * D + 16 * i + 8 * hf);
            }
            x1[n][i] = __builtin_bit_cast(bf16x8, v1);
            x2[n][i] = __builtin_bit_cast(bf16x8, v2);
        }
        if (KEYS) {
            lo[n] = s.causal ? t - shift : 0;
            hi[n] = live ? Q.len - 1 : -1;
        } else {
            lo[n] = 0;
            hi[n] = live ? (s.causal ? min(K.len - 1, t + shift) : K.len - 1) : -1;
            // d = sum dO O, and lse in powers of two
            float d = 0.0f;
            lse2[n] = INFINITY;
            if (live) {
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
                        d = __builtin_fmaf((float)x2[n][i][j], o[j], d);
                }
            }
            d += __shfl_xor(d, 32);
            delta[n] = d;
            if (live) {
                const int64_t at = head * s.qrows + Q.first + t;
                const float l = a.lse[at];
                lse2[n] = l == -INFINITY ? INFINITY : l * LOG2E;
                if (part == 0 && hf == 0) {
                    a.sums[at] = lse2[n];
                    a.sums[s.H * s.qrows + at] = d;
                }
            }
        }
    }
    // tiles [first, first + tiles) of streamed rows, for keys of each head in turn
    int first = 0, tiles;
    if (KEYS) {
        first = s.causal ? max(0, row0 - shift) / BT : 0;
        tiles = row0 < K.len ? max(0, (Q.len + BT - 1) / BT - first) : 0;
    } else {
        const int tmax = min((row0 + KEEP<NS> - 1) / G, Q.len - 1);
        const int keys = Q.len > row0 / G
                             ? max(0, (s.causal ? min(K.len - 1, tmax + shift) : K.len - 1) + 1)
                             : 0;
        tiles = (keys + BT - 1) / BT;
    }
    const int64_t all = (int64_t)tiles * (KEYS ? G : 1);
    const int j0 = (int)(all * part / parts), j1 = (int)(all * (part + 1) / parts);
    // streamed rows that need no mask
    const int free_lo = KEYS && s.causal ? wrow + 32 * NS - 1 - shift : 0;
    const int free_hi = KEYS ? Q.len - 1
                             : (s.causal ? min(K.len - 1, wrow / G + shift) : K.len - 1);

    const int64_t ld1 = KEYS ? s.ldq : s.ldk, ld2 = KEYS ? a.lddo : s.ldv;
    TileLoad<D, BT, THREADS> load1, load2;
    load1.init(ld1, tid);
    load2.init(ld2, tid);
    auto tile_of = [&](int j, int &head) {
        const int g = KEYS ? j / tiles : 0;
        head = KEYS ? hk * G + g : hk;
        return first + j - g * tiles;
    };
    auto fetch = [&](int j, uint8_t *buf) {
        int head;
        const int r0 = tile_of(j, head) * BT, left = (KEYS ? Q.len : K.len) - r0;
        const int64_t at = (KEYS ? Q.first : K.first) + r0;
        const uint16_t *p1 = (KEYS ? s.q : s.k) + at * ld1 + head * D;
        const uint16_t *p2 = (KEYS ? a.dO : s.v) + at * ld2 + head * D;
        load1.issue(reinterpret_cast<const uint8_t *>(p1), left, ld1, buf, tid);
        load2.issue(reinterpret_cast<const uint8_t *>(p2), left, ld2, buf + TILE, tid);
        if (KEYS && wave < 2) {
            const float *sums = a.sums + (int64_t)wave * s.H * s.qrows + head * s.qrows + at;
            dma_load4_at(sums + min(lane, left - 1), dma_lds(buf + 2 * TILE + wave * 256));
        }
    };

    f32x16 acc1[NS][DT], acc2[KEYS ? NS : 1][KEYS ? DT : 1];
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                acc1[n][d][r] = 0.0f;
                if (KEYS)
                    acc2[n][d][r] = 0.0f;
            }

    auto block = [&](auto maskc, const uint8_t *buf, int sub, int r0) {
        constexpr bool MASK = decltype(maskc)::value;
        const uint8_t *t1 = buf, *t2 = buf + TILE;
        f32x16 sc[NS], dp[NS];
        const f32x16 zero = {};
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            const bf16x8 w = row_operand<D>(t1, 32 * sub + l32, i, hf);
#pragma unroll
            for (int n = 0; n < NS; ++n)
                sc[n] = mfma(w, x1[n][i], i == 0 ? zero : sc[n]);
        }
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            const bf16x8 w = row_operand<D>(t2, 32 * sub + l32, i, hf);
#pragma unroll
            for (int n = 0; n < NS; ++n)
                dp[n] = mfma(w, x2[n][i], i == 0 ? zero : dp[n]);
        }
        f32x4_t ls[4], dl[4];  // of streamed queries 8 e + 4 hf + 0 .. 3
        if (KEYS) {
            const float *const f = reinterpret_cast<const float *>(buf + 2 * TILE) + 32 * sub + 4 * hf;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ls[e] = *reinterpret_cast<const f32x4_t *>(f + 8 * e);
                dl[e] = *reinterpret_cast<const f32x4_t *>(f + 64 + 8 * e);
            }
        }
        bf16x8 pb[NS][2], sb[NS][2];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int from = lo[n] - r0 - 32 * sub - 4 * hf, to = hi[n] - r0 - 32 * sub - 4 * hf;
#pragma unroll
            for (int ch = 0; ch < 2; ++ch) {
                uint32_t pw[4], sw[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p[2], ds[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int r = 8 * ch + 2 * e + k, x = 8 * (r >> 2) + (r & 3);
                        p[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(
                            sc[n][r], c, -(KEYS ? ls[r >> 2][r & 3] : lse2[n])));
                        ds[k] = p[k] * (dp[n][r] - (KEYS ? dl[r >> 2][r & 3] : delta[n]));
                        if (MASK) {
                            const bool in = x <= to && (!KEYS || x >= from);
                            p[k] = in ? p[k] : 0.0f;
                            ds[k] = in ? ds[k] : 0.0f;
                        }
                    }
                    pw[e] = pack_bf16(p[0], p[1]);
                    sw[e] = pack_bf16(ds[0], ds[1]);
                }
                pb[n][ch] = __builtin_bit_cast(bf16x8, u32x4{pw[0], pw[1], pw[2], pw[3]});
                sb[n][ch] = __builtin_bit_cast(bf16x8, u32x4{sw[0], sw[1], sw[2], sw[3]});
            }
        }
#pragma unroll
        for (int ch = 0; ch < 2; ++ch)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const bf16x8 w1 = transposed_operand<D>(t1, 2 * sub + ch, d, lane);
#pragma unroll
                for (int n = 0; n < NS; ++n)
                    acc1[n][d] = mfma(w1, sb[n][ch], acc1[n][d]);
                if constexpr (KEYS) {
                    const bf16x8 w2 = transposed_operand<D>(t2, 2 * sub + ch, d, lane);
#pragma unroll
                    for (int n = 0; n < NS; ++n)
                        acc2[n][d] = mfma(w2, pb[n][ch], acc2[n][d]);
                }
            }
    };

    // At the start of a step its tile's loads (the last issued) have landed and every
    // wavefront has finished the step before it, whose buffer takes the next tile.
    if (j0 < j1)
        fetch(j0, lds);
    for (int j = j0; j < j1; ++j) {
        const uint8_t *const buf = lds + ((j - j0) & 1) * BUF;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (j + 1 < j1)
            fetch(j + 1, lds + ((j - j0 + 1) & 1) * BUF);
        int head;
        const int r0 = tile_of(j, head) * BT;
#pragma unroll 1
        for (int sub = 0; sub < SUB; ++sub) {
            const int from = r0 + 32 * sub;
            if (from >= free_lo && from + 31 <= free_hi)
                block(Flag<false>{}, buf, sub, r0);
            else
                block(Flag<true>{}, buf, sub, r0);
        }
    }

    // channel 32 d + 8 e + 4 hf + r % 4 of the lane's row; padding rows: zeros
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        const int row = wrow + 32 * n + l32;
        const int t = KEYS ? row : row / G, head = KEYS ? hk : hk * G + row - t * G;
        if (t >= (KEYS ? K.cap : Q.cap))
            continue;
        const bool live = t < (KEYS ? K.len : Q.len);
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
            store(acc1[n], a.dk, a.lddk, a.part, a.scale);
            store(acc2[n], a.dv, a.lddv, a.part + (int64_t)parts * s.B * s.Hk * rows * D, 1.0f);
        } else {
            store(acc1[n], a.dq, a.lddq, a.part, a.scale);
        }
    }
}

// Partial sums added in order, 4 channels a thread (blockIdx.y: dk, dv).
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
    const int b = unit / s.Hk, hk = unit - b * s.Hk;
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
    const int64_t o = (R.first + t) * (!KEYS ? a.lddq : blockIdx.y ? a.lddv : a.lddk) + head * D + ch;
    if (a.bf16)
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(out) + o) =
            u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(out) + o) = v;
}

int64_t blocks(const SeqAttn &s, bool keys)
{
    const int64_t rows = keys ? s.KT : (int64_t)s.T * (s.H / s.Hk);
    return (rows + KEEP<1> - 1) / KEEP<1> * s.B * s.Hk;
}

template <int D, bool KEYS>
hipError_t go(const SeqAttnGrad &a, hipStream_t stream)
{
    const int parts = KEYS ? a.kparts : a.qparts;
    const unsigned grid = (unsigned)(blocks(a.s, KEYS) * parts);
    if (grid)
        hipLaunchKernelGGL((seq_attn_grad_kernel<D, KEYS, 1, D == 64 ? 64 : 32>), dim3(grid),
                           dim3(THREADS), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts < 2 || !grid)
        return e;
    const int64_t rows = KEYS ? a.s.KT : (int64_t)a.s.T * (a.s.H / a.s.Hk);
    const int64_t threads = (int64_t)a.s.B * a.s.Hk * rows * (D / 4);
    hipLaunchKernelGGL((attn_grad_join_kernel<D, KEYS>),
                       dim3((unsigned)((threads + 255) / 256), KEYS ? 2 : 1), dim3(256), 0, stream,
                       a);
    return hipGetLastError();
}

}  // namespace

SeqAttnGradPlan seq_attn_grad_plan(const SeqAttn &s, bool keys, int cus)
{
    auto parts = [&](int64_t wgs, int64_t tiles) {
        if (wgs == 0 || wgs >= cus)
            return 1;
        const int64_t want = (cus + wgs - 1) / wgs, most = tiles / 4;
        return (int)(most < 2 ? 1 : want < most ? want : most);
    };
    const int64_t bt = s.dh == 64 ? 64 : 32;
    SeqAttnGradPlan p{1, 1};
    p.qparts = parts(blocks(s, false), (s.KT + bt - 1) / bt);
    if (keys)
        p.kparts = parts(blocks(s, true), (s.T + bt - 1) / bt * (s.H / s.Hk));
    return p;
}

int64_t seq_attn_grad_workgroups(const SeqAttn &s, const SeqAttnGradPlan &p)
{
    const int64_t q = blocks(s, false) * p.qparts, k = blocks(s, true) * p.kparts;
    return q > k ? q : k;
}

size_t seq_attn_grad_bytes(const SeqAttn &s, const SeqAttnGradPlan &p)
{
    const size_t sums = ((size_t)2 * s.H * s.qrows * 4 + 255) & ~(size_t)255;
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
    a.part = a.sums + (((size_t)2 * a.s.H * a.s.qrows * 4 + 255) & ~(size_t)255) / 4;
    const hipError_t e = a.s.dh == 64 ? go<64, false>(a, stream) : go<128, false>(a, stream);
    if (e != hipSuccess || !a.dk)
        return e;
    return a.s.dh == 64 ? go<64, true>(a, stream) : go<128, true>(a, stream);
}

}  // namespace qlk
