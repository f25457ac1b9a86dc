/*
 * qlinear_block.h — the operators of a transformer block around its quantized
 * linears (qlinear.h, whose conventions apply to every function here): 4-bit
 * microscaled arithmetic, the gated feed-forward with its backward pass, and
 * rotary positions.
 */
#ifndef QLINEAR_BLOCK_H
#define QLINEAR_BLOCK_H

#include "qlinear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- MXFP4 ------------------------------------------------------------------
 *
 * QL_FMT_MXFP4 weights (qlinear.h) go through qlinear_quantize and every
 * forward and block_forward function like the other formats.  Below: the size
 * of their scales, the compressed formats read back, and the product with
 * activations that are MXFP4 too. */

/* Bytes of the scales of an N x K MXFP4 tensor: N * (K/32).  0 when K % 32 != 0
 * or a size is non-positive. */
size_t qlinear_mx_scales_bytes(int64_t N, int64_t K);

/* W[N][K] = code * scale of QL_FMT_MXFP4, QL_FMT_Q4 or QL_FMT_INT8 codes (16-byte
 * aligned) and scales, as fp32 (exact) or bf16 (wdt; exact for MXFP4, otherwise
 * rounded to nearest even; 16-byte aligned W).  N * K < 2^40.  N == 0 is a
 * no-op.  Asynchronous. */
int qlinear_dequantize(int fmt, const void *codes, const void *scales, int64_t N, int64_t K,
                       void *W, int wdt, hipStream_t stream);

/* Activations X [M][K] (fp32 or bf16, 16-byte aligned, K % 32 == 0) as MXFP4:
 * qx uint8 [M][K/2] (16-byte aligned) and sx uint8 [M][K/32], by the rule of
 * QL_FMT_MXFP4 weights.  A block holding a NaN or Inf gets the NaN scale 255 and
 * zero codes: there is no synchronous status.  M * K < 2^40, M < 2^31.
 * Asynchronous; M == 0 is a no-op. */
int qlinear_mx_quantize_act(const void *X, int xdt, int64_t M, int64_t K, uint8_t *qx,
                            uint8_t *sx, hipStream_t stream);

/* Y = the product of MXFP4 activations (qx 16-byte aligned, sx) and MXFP4
 * weights (codes 16-byte aligned, scales) on the 4-bit matrix cores, with fp32
 * accumulation, then the epilogue ep (NULL: none, fp32 Y).  Asynchronous; Y
 * must not alias an input (except ep->residual as for qlinear_forward_ep).
 * Errors as qlinear_forward_ep. */
int qlinear_mx_forward(const uint8_t *qx, const uint8_t *sx, int64_t M, int64_t K,
                       const void *codes, const uint8_t *scales, int64_t N, void *Y,
                       const ql_epilogue *ep, hipStream_t stream);

/* ---- gated feed-forward -----------------------------------------------------
 *
 * The first half of a gated feed-forward block, both projections, the
 * activation and the product in one kernel:
 *
 *     G = X Wg^T + bg,  U = X Wu^T + bu,  H[m][n] = act(G[m][n]) * U[m][n]
 *
 * (the second half is a linear layer on H).  Weights: QL_FMT_MXFP4, QL_FMT_Q4 or
 * QL_FMT_INT8, both of one format, [N][K]; X bf16 [M][K]; act QL_ACT_NONE,
 * QL_ACT_GELU (exact form) or QL_ACT_SILU.  G and U stay in fp32; MXFP4 weights
 * enter exactly, q4 and int8 weights c * s exactly or as the sum of two bf16 (off by
 * at most 2^-22 of each q4 weight, 2^-16 of each int8 weight).  An infinite
 * activation gives an infinity of the product's sign, NaN for a weight of zero;
 * finite ones of q4 and int8 pairs: up to 7e34 in size (as in qlinear.h).
 * Alignment: X and codes 16 bytes, fp16 scales 2, biases 4. */
typedef struct {
    int fmt;                     /* ql_fmt */
    const uint16_t *X;           /* bf16 [M][K] */
    int64_t M, K, N;
    const void *gate_codes, *gate_scales;
    const void *up_codes, *up_scales;
    const float *gate_bias, *up_bias;  /* fp32 [N], each may be NULL */
    int act;                     /* ql_act */
} ql_gated;

/* H [M][N], fp32 (4-byte aligned) or bf16 (2-byte) as hdt says; it must not
 * alias an input.  M == 0 is a no-op.  M, N < 2^31, K < 2^22 (QL_ERR_UNSUPPORTED
 * otherwise).  Asynchronous. */
int qlinear_gated_forward(const ql_gated *g, void *H, int hdt, hipStream_t stream);

/* The backward pass.  From dH, the gradient of H, and the forward's inputs (G
 * and U are formed again, nothing is kept from the forward pass):
 *
 *     dU = dH act(G),  dG = dH U act'(G)          bf16, each rounded once
 *     dX = dG Wg + dU Wu
 *     dWg = dG^T X,  dWu = dU^T X
 *     dbg[n] = sum_m dG[m][n],  dbu[n] = sum_m dU[m][n]
 *
 * with fp32 accumulation from the bf16 dG and dU.  dWg and dWu are the
 * gradients of the weights' values (quantization-aware training passes them on
 * as they are; adapters on frozen weights take dG and dU).  In dX, weights enter
 * as in the forward pass.  Results do not depend on
 * anything but the inputs: every sum has one order. */
typedef struct {
    const void *dH;              /* [M][N], fp32 or bf16 as dhdt says */
    int dhdt;                    /* ql_dtype */
    uint16_t *dG, *dU;           /* bf16 [M][N], 16-byte aligned, required */
    void *dX;                    /* [M][K], dtype dxdt, 16-byte aligned; or NULL */
    int dxdt;
    void *dWg, *dWu;             /* [N][K], dtype dwdt, 16-byte aligned; both or neither */
    int dwdt;
    float *dbg, *dbu;            /* fp32 [N], each may be NULL */
} ql_gated_grad;

/* No output may alias an input or another output (the same address:
 * QL_ERR_INVALID).  N % 8 == 0 and K % 32 == 0;
 * M == 0 writes zeros to dW and db and nothing else.  Workspace (per stream, as
 * in qlinear.h): for dX above 512 rows, or where K % 128 != 0 or a scale tensor is
 * not 4-byte aligned, the weights in bf16 (4 N K bytes; q4, int8: 8), and fp32
 * partial sums where few tiles make the products split their reductions (at most
 * 256 MiB).
 * Sizes: M, N, K < 2^22 and M, N times K < 2^40 (QL_ERR_UNSUPPORTED otherwise).
 * Asynchronous. */
int qlinear_gated_backward(const ql_gated *g, const ql_gated_grad *d, hipStream_t stream);

/* ---- rotary positions -------------------------------------------------------
 *
 * Of each of the `heads` heads of dh channels (head h at column h * dh of a row:
 * the query and key heads of a fused QKV output in one call), the pairs (a, b) =
 * (x[j], x[j + rot/2]) (half layout) or (x[2j], x[2j + 1]) (interleaved), j <
 * rot / 2, become
 *
 *     (m (a cos t - b sin t), m (b cos t + a sin t)),   t = position * freqs[j]
 *
 * with m = mscale, and the channels from rot on stay as they are.  adjoint != 0
 * turns by -t: the gradient of x from that of the output.  Row r's position is
 * positions[r], or start + r % period when positions is NULL (sequences of
 * `period` rows).  freqs: device fp64 [rot/2], radians per position, where a
 * longer context's scaling enters; the angle is the exact product, reduced before it
 * is rounded (positions up to 2^31 in size).  x, o: rows of ldx, ldo elements, fp32 or bf16 (dt, both), x ==
 * o with ldx == ldo for in place, otherwise no element of both (QL_ERR_INVALID; other
 * columns of the same rows may be); aligned to an element.
 * rot even, 2 <= rot <= dh; heads * dh <= ldx, ldo < 2^31; rows < 2^24.
 * Asynchronous; rows == 0 is a no-op. */
int qlinear_rotary(const void *x, int64_t ldx, void *o, int64_t ldo, int dt, int64_t rows,
                   int64_t heads, int64_t dh, int64_t rot, const double *freqs,
                   const int64_t *positions, int64_t start, int64_t period, float mscale,
                   int interleaved, int adjoint, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* QLINEAR_BLOCK_H */
