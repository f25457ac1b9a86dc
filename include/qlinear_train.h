/*
 * qlinear_train.h — the normalisation and the masked attention of a transformer
 * block, each with its backward pass (qlinear.h's conventions apply to every function
 * here; the linears are there, the gated feed-forward and rotary positions in
 * qlinear_block.h).
 */
#ifndef QLINEAR_TRAIN_H
#define QLINEAR_TRAIN_H

#include "qlinear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- normalisation ----------------------------------------------------------
 *
 * A block's root-mean-square normalisation with the residual's addition: by row,
 *
 *     v = x + res                       one fp32 rounding (res NULL: v = x)
 *     h = v                             the new residual stream, in res's dtype
 *     y = v weight / sqrt(mean(v^2) + eps)
 *
 * x, res, h and y: rows of ldx, ldr, ldh, ldy >= N elements, fp32 or bf16 (h as res:
 * rdt, also where res is NULL), aligned to an element.  weight fp32 [N] or NULL (ones).
 * y is formed from v before its rounding to h's dtype, as the fp32 nearest to the
 * exact value (a few fp64 roundings off a tie), for bf16 rounded again.  qx int8
 * [M][N], sx fp16 [M]: the int8 activations of qlinear_forward_w8a8, as
 * qlinear_quantize_act gives them for the fp32 y (N % 32 == 0, qx 16-byte aligned).
 * h, y, and qx with sx may each be NULL, not all.  h or y may be x or res in place
 * (same address, dtype and ld); no output shares elements with another argument
 * otherwise (QL_ERR_INVALID; other columns of the same rows may be).  eps >= 0; a row of
 * zeros has y = 0, also with eps = 0.  N <= 16384, M < 2^24 (QL_ERR_UNSUPPORTED).
 * Asynchronous; M == 0 is a no-op. */
typedef struct {
    const void *x;
    int64_t ldx;
    int xdt;                     /* ql_dtype */
    const void *res;
    int64_t ldr;
    int rdt;                     /* of res and h */
    const float *weight;
    double eps;
    int64_t M, N;
    void *h;
    int64_t ldh;
    void *y;
    int64_t ldy;
    int ydt;
    int8_t *qx;
    uint16_t *sx;
} ql_norm;

int qlinear_rms_norm(const ql_norm *n, hipStream_t stream);

/* Its backward pass from dy, the gradient of y, and h, the normalised values (the v
 * above, or their rounding that was kept):
 *
 *     dx = dres + r (g - u mean(g u)),  dw = sum over rows of dy u,
 *          r = 1 / sqrt(mean(h^2) + eps),  u = h r,  g = dy weight
 *
 * (r = 0 for a row of zeros with eps = 0: dx = dres, and nothing for dw.)
 * dx, the gradient of x and of res alike; dres: the one that arrives at h from further
 * on (NULL: 0), of dx's dtype.  dw fp32 [N] or NULL.  dx may be dy, h or dres in place
 * (same address, dtype and ld); other conventions as above.  Sums of a row in
 * fp64; dw in one fixed order, fp32 over some of the rows and fp64 over these sums.
 * Workspace with dw (per stream, as in qlinear.h): at most 12 N bytes per CU.  M == 0
 * writes zeros to dw and nothing else. */
typedef struct {
    const void *dy;
    int64_t lddy;
    int dydt;                    /* ql_dtype */
    const void *h;
    int64_t ldh;
    int hdt;
    const void *dres;
    int64_t lddres;
    const float *weight;
    double eps;
    int64_t M, N;
    void *dx;
    int64_t lddx;
    int dxdt;                    /* of dx and dres */
    float *dw;
} ql_norm_grad;

int qlinear_rms_norm_backward(const ql_norm_grad *g, hipStream_t stream);

/* ---- masked attention --------------------------------------------------------
 *
 * Softmax attention of B sequences, of up to Tq queries and Tk keys: for query i of a
 * sequence with n queries and m keys, and each of the H query heads (dh channels, 64
 * or 128; head h at column h * dh of its row), which share Hk key heads (H % Hk == 0;
 * query head h reads key head h / (H / Hk)),
 *
 *     O_i = sum_j P_ij V_j,  P_ij = exp(s_ij - lse_i),  s_ij = scale * <Q_i, K_j>,
 *     lse_i = log sum_j exp(s_ij)
 *
 * over the keys j < m, with causal only those up to i + m - n (the last query sees
 * every key).  A query that sees no key has O = 0 and lse = -infinity.
 *
 * Where a sequence's rows lie, for queries (q, O, lse: q_rows rows) and keys (k, v:
 * k_rows rows) each: Tq (Tk) rows from b * Tq on; or with offsets (device, [B + 1], not
 * decreasing) those from offsets[b] up to offsets[b + 1], Tq (Tk) of them at most.  With
 * lens (device, [B]) the first lens[b] of these rows are the sequence's and the others
 * padding: never read, written as zeros (lse: -infinity).  Rows of no sequence stay as
 * they are.  Offsets and lens are read on the device; values that lie outside of a
 * tensor or a sequence's place are cut to it.  Sequences that share query rows (in the
 * backward pass, query or key rows) leave one of their results there, or a mixture.
 *
 * q, k, v: bf16, 16-byte aligned, rows of ldq, ldk, ldv elements (% 8 == 0, < 2^24).  O:
 * fp32 (16-byte aligned) or bf16 (8-byte), rows of ldo (% 4 == 0).  scale: 0 (taken as
 * 1e-30) or 1e-30 to 2.3e38; scores times log2(e) that leave fp32's range give NaN.  The
 * probabilities enter the product with V rounded to bf16, sums are fp32.  Values that are not
 * finite keep to what they are part of, but not under a causal mask alone: there a key
 * may reach queries up to 255 before those that see it, and in the backward pass a query
 * the gradients of keys up to 255 behind those it sees (0 * infinity).  Sizes: B * H * Tq,
 * B * Hk * Tk < 2^31, Tk <= 2^30, B * Hk * ceil(Tq * H / Hk / 32) < 2^24, in the backward
 * pass B * Hk * ceil(Tk / 128) < 2^24 too (QL_ERR_UNSUPPORTED). */
typedef struct {
    const uint16_t *q;
    int64_t ldq;
    const uint16_t *k;
    int64_t ldk;
    const uint16_t *v;
    int64_t ldv;
    int64_t q_rows, k_rows;
    const int64_t *q_offsets, *k_offsets;  /* device, or NULL */
    const int64_t *q_lens, *k_lens;        /* device, or NULL */
    int64_t B, Tq, Tk, H, Hk, dh;
    int causal;
    float scale;
} ql_attn;

/* O, and with lse (fp32 [H][q_rows], or NULL) what the backward pass takes.  O and lse
 * share no elements with an input (QL_ERR_INVALID).  Workspace (per stream, as in
 * qlinear.h) where few queries leave CUs idle: fp32 partial results of parts of the
 * keys, at most 80 MiB.  Asynchronous; B == 0 or Tq == 0 is a no-op. */
int qlinear_attention_forward(const ql_attn *a, void *o, int64_t ldo, int odt, float *lse,
                              hipStream_t stream);

/* The backward pass, from O and lse of qlinear_attention_forward on the same inputs and
 * dO, the gradient of O:
 *
 *     dV_j = sum_i P_ij dO_i,  dS_ij = P_ij (<dO_i, V_j> - <dO_i, O_i>),
 *     dQ_i = scale sum_j dS_ij K_j,  dK_j = scale sum_i dS_ij Q_i
 *
 * (K_j and V_j: summed over the query heads that share them.)  The probabilities are
 * formed again from lse; P and dS enter the products rounded to bf16 (in sums over few
 * rows, and for outputs of few, as two bf16), sums are fp32 in one fixed order.  <dO, O> is as exact as the O that
 * was kept (over up to 128 keys it is formed anew): where a row's probability is that of a
 * few keys, dS is much smaller than its terms and a bf16 O is most of its error.  Errors
 * of dq and dk relative to their norm, of bf16 gradients: scores of a spread of 1, 4, 10
 * and 30 up to 0.0025, 0.0038, 0.0059 and 0.0075 with a bf16 O, 0.0025, 0.0030, 0.0034 and
 * 0.0034 with an fp32 O (the gradients' own rounding: 0.0017).  dq of a query that sees
 * one key, and dk of a sequence's only key, are 0.  dO: bf16, 16-byte aligned, rows of
 * lddo (% 8 == 0, < 2^24).  dq, dk, dv: dtype dt, aligned and strided as O; dk and dv both
 * or neither.  Rows as above: padding rows of q (k, v) get zeros in dq (dk, dv), those of no sequence stay.  No output
 * shares elements with an input or another output (QL_ERR_INVALID; other columns of the
 * same rows may be: the gradients may be those of a fused QKV output).  Workspace (per
 * stream, as in qlinear.h): 16 H q_rows bytes, and fp32 partial sums where few rows leave
 * CUs idle, at most 160 MiB.  Asynchronous. */
typedef struct {
    const void *o;
    int64_t ldo;
    int odt;                     /* ql_dtype */
    const float *lse;
    const uint16_t *dO;
    int64_t lddo;
    void *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    int dt;                      /* of dq, dk and dv */
} ql_attn_grad;

int qlinear_attention_backward(const ql_attn *a, const ql_attn_grad *g, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* QLINEAR_TRAIN_H */
