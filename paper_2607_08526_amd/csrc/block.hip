// C-ABI entry points of include/qlinear_block.h: argument checks, choice of
// kernel and launches.  Every check happens before anything is enqueued; no
// entry point throws or aborts.
#include <algorithm>

#include "epilogue.h"
#include "internal.h"
#include "qlinear_block.h"

using namespace qlk;

namespace {

constexpr int64_t I31 = (int64_t)1 << 31, I22 = (int64_t)1 << 22, I40 = (int64_t)1 << 40;

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

bool dt_ok(int dt) { return dt == QL_DT_F32 || dt == QL_DT_BF16; }

bool fmt_ok(int f) { return f == QL_FMT_MXFP4 || f == QL_FMT_Q4 || f == QL_FMT_INT8; }

// a * b >= limit, for a, b >= 0
bool product_reaches(int64_t a, int64_t b, int64_t limit) { return b > 0 && a >= (limit + b - 1) / b; }

// whether rows of w elements (of `size` bytes) at strides ldx and ldo share any, the
// same rows in the same place (in place) left out
bool rows_overlap(const void *x, int64_t ldx, const void *o, int64_t ldo, int64_t rows, int64_t w,
                  uintptr_t size)
{
    const uintptr_t a = (uintptr_t)x, b = (uintptr_t)o;
    if (a == b)
        return rows > 1 && ldx != ldo;
    if (a >= b + (uintptr_t)((rows - 1) * ldo + w) * size ||
        b >= a + (uintptr_t)((rows - 1) * ldx + w) * size)
        return false;
    // columns of one buffer: apart in every row, or not
    if (rows == 1 || ldx != ldo)
        return true;
    const int64_t apart = (int64_t)((a > b ? a - b : b - a) / size) % ldx;
    return apart < w || ldx - apart < w;
}

int status(hipError_t e) { return e == hipSuccess ? QL_OK : QL_ERR_HIP; }

int check_gated(const ql_gated *g)
{
    if (!g || !fmt_ok(g->fmt) ||
        (g->act != QL_ACT_NONE && g->act != QL_ACT_GELU && g->act != QL_ACT_SILU))
        return QL_ERR_INVALID;
    if (g->M < 0 || g->N <= 0 || g->K <= 0 || g->K % QL_BLOCK)
        return QL_ERR_SHAPE;
    if (g->M >= I31 || g->N >= I31 || g->K >= I22)
        return QL_ERR_UNSUPPORTED;
    if (!g->gate_codes || !g->gate_scales || !g->up_codes || !g->up_scales || (g->M > 0 && !g->X))
        return QL_ERR_INVALID;
    const uintptr_t sa = g->fmt == QL_FMT_MXFP4 ? 1 : 2;
    if (!aligned(g->gate_codes, 16) || !aligned(g->up_codes, 16) || !aligned(g->gate_scales, sa) ||
        !aligned(g->up_scales, sa) || !aligned(g->gate_bias, 4) || !aligned(g->up_bias, 4) ||
        !aligned(g->X, 16))
        return QL_ERR_ALIGN;
    return QL_OK;
}

GateArgs gate_args(const ql_gated &g)
{
    GateArgs t{};
    t.bias[0] = g.gate_bias;
    t.bias[1] = g.up_bias;
    t.act = g.act;
    return t;
}

// the two projections of a gated pair with the outputs t
int launch_gated(const ql_gated &g, const GateArgs &t, hipStream_t stream)
{
    int shape;
    const RowsKernel kernel = choose_rows(g.fmt, false, true, g.M, g.M, g.N, g.K, current_cus(),
                                          &shape);
    if (kernel == ROWS_ANY && rows_tiles(g.M, g.N, true) > MAX_WORKGROUPS)
        return QL_ERR_UNSUPPORTED;
    if (kernel == ROWS_TILE) {
        TileArgs a{};
        a.X = g.X;
        a.planes = 1;
        a.codes[0] = (const uint8_t *)g.gate_codes;
        a.codes[1] = (const uint8_t *)g.up_codes;
        a.scales[0] = g.gate_scales;
        a.scales[1] = g.up_scales;
        a.gate = t;
        a.M = (int)g.M;
        a.N = (int)g.N;
        a.K = (int)g.K;
        a.rows = shape;
        return status(launch_qgemm_tile(g.fmt, a, stream));
    }
    RowsGroup r{};
    RowsArgs &d = r.d[0];
    d.X = g.X;
    d.codes[0] = (const uint8_t *)g.gate_codes;
    d.codes[1] = (const uint8_t *)g.up_codes;
    d.scales[0] = g.gate_scales;
    d.scales[1] = g.up_scales;
    d.gate = t;
    d.M = (int)g.M;
    d.N = (int)g.N;
    d.K = (int)g.K;
    d.shape = shape;
    r.n = 1;
    r.maxM = (int)g.M;
    return status(kernel == ROWS_KGM ? launch_qgemm_kgm(g.fmt, false, r, stream)
                                     : launch_qgemm_rows(g.fmt, false, r, stream));
}

// gemm_dx's costs by planes (MXFP4; q4, int8) and rows of a tile (128, 64).  Measured,
// us of dX in 128 / 64 rows, N = 2752, K = 1024: MXFP4 107 rows 20.2 / 18.1, 400 rows 26.0
// / 24.8; q4 107 rows 25.2 / 23.6, 400 rows 32.2 / 35.0.
constexpr GemmCost DX_COST[2][2] = {{{0.55, 0.55}, {0.45, 0.40}}, {{1.0, 1.0}, {0.87, 0.87}}};

// gemm_bf16's by rows of a tile (128, 64), fitted to 78 products in 1 to 8 parts of both
// (the choice takes 1.015 times the best one's time on average, 1.05 at the ninth decile).
// Measured, us in 128 / 64 rows: dW 2048 rows of 2048 x 1024 38.5 / 29.5, of 4096 x 1536
// 54.4 / 64.2, of 5504 x 2048 96 / 113; dX 2048 rows of 1024 x 1024 33.0 / 31.0; and in 2 /
// 5 parts of 128 rows dX 2048 rows of 4096 x 1536 81.9 / 72.2.
constexpr GemmCost BF16_COST[2] = {{0.48, 0.38}, {0.34, 0.25}};

// the rows of a tile and the parts estimated to be fastest for outputs R x S of a
// reduction of C; cost: of tiles of 128 and 64 rows
void gemm_plan(int64_t R, int64_t S, int64_t C, int problems, const GemmCost *cost, int cus,
               int &rows, int &parts)
{
    constexpr int64_t PART_BYTES = (int64_t)256 << 20;  // of partial sums
    double best = 0.0;
    for (int h = 0; h < 2; ++h) {
        const int tile = h ? 64 : 128;
        double us;
        const int64_t p = gemm_parts(gemm_tiles(tile, R, S) * problems, R * problems, S, C,
                                     cost[h], cus, &us);
        if (h == 0 || us < best) {
            best = us;
            rows = tile;
            parts = (int)std::max<int64_t>(1, std::min(p, PART_BYTES / (problems * R * S * 4)));
        }
    }
}

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

}  // namespace

namespace qlk {

GradPlan grad_plan(int fmt, int64_t M, int64_t N, int64_t K, const void *scales0,
                   const void *scales1, bool dx, bool dw, int cus)
{
    GradPlan g{false, 1, 128, 1, 128};
    const int planes = fmt == QL_FMT_MXFP4 ? 1 : 2;
    // dX straight from the compressed weights up to a few hundred rows, beyond from
    // a bf16 copy (us of dX at N = 4096, mxfp4 / q4: 128 rows of K = 1536 21.9 / 27.8
    // against 28.8 / 36.0, 1024 rows of K = 2048 61.6 / 89.2 against 58.2 / 90.6)
    g.direct = M <= 512 && dx_takes(K, scales0, scales1);
    if (dx && g.direct)
        gemm_plan(M, K, 2 * N, 1, DX_COST[planes - 1], cus, g.xrows, g.xparts);
    else if (dx)
        gemm_plan(M, K, 2 * planes * N, 1, BF16_COST, cus, g.xrows, g.xparts);
    if (dw)
        gemm_plan(N, K, M, 2, BF16_COST, cus, g.wrows, g.wparts);
    return g;
}

}  // namespace qlk

extern "C" {

size_t qlinear_mx_scales_bytes(int64_t N, int64_t K)
{
    if (N <= 0 || K <= 0 || K % QL_BLOCK)
        return 0;
    return (size_t)N * (size_t)(K / QL_BLOCK);
}

int qlinear_dequantize(int fmt, const void *codes, const void *scales, int64_t N, int64_t K,
                       void *W, int wdt, hipStream_t stream)
{
    if (!fmt_ok(fmt) || !dt_ok(wdt))
        return QL_ERR_INVALID;
    if (N < 0 || K <= 0 || K % QL_BLOCK)
        return QL_ERR_SHAPE;
    if (product_reaches(N, K, I40))
        return QL_ERR_UNSUPPORTED;
    if (N == 0)
        return QL_OK;
    if (!codes || !scales || !W)
        return QL_ERR_INVALID;
    if (!aligned(codes, 16) || !aligned(scales, fmt == QL_FMT_MXFP4 ? 1 : 2) || !aligned(W, 16))
        return QL_ERR_ALIGN;
    const DequantJob job{codes, scales, W, nullptr};
    return status(launch_dequantize(fmt, &job, 1, N, K, wdt == QL_DT_BF16, stream));
}

int qlinear_mx_quantize_act(const void *X, int xdt, int64_t M, int64_t K, uint8_t *qx, uint8_t *sx,
                            hipStream_t stream)
{
    if (!dt_ok(xdt))
        return QL_ERR_INVALID;
    if (M < 0 || K <= 0 || K % QL_BLOCK)
        return QL_ERR_SHAPE;
    if (M >= I31 || product_reaches(M, K, I40))
        return QL_ERR_UNSUPPORTED;
    if (M == 0)
        return QL_OK;
    if (!X || !qx || !sx)
        return QL_ERR_INVALID;
    if (!aligned(X, 16) || !aligned(qx, 16))
        return QL_ERR_ALIGN;
    return status(launch_mx_quantize(X, xdt == QL_DT_BF16, M, K, qx, sx, nullptr, stream));
}

int qlinear_mx_forward(const uint8_t *qx, const uint8_t *sx, int64_t M, int64_t K,
                       const void *codes, const uint8_t *scales, int64_t N, void *Y,
                       const ql_epilogue *ep, hipStream_t stream)
{
    if (ep) {
        const int st = epilogue_status(*ep, Y);
        if (st != QL_OK)
            return st;
    }
    if (M < 0 || N <= 0 || K <= 0 || K % QL_BLOCK)
        return QL_ERR_SHAPE;
    if (M >= I31 || N >= I31 || K >= I31)
        return QL_ERR_UNSUPPORTED;
    if (!codes || !scales || (M > 0 && (!qx || !sx || !Y)))
        return QL_ERR_INVALID;
    if (!aligned(codes, 16) ||
        (M > 0 && (!aligned(qx, 16) || !aligned(Y, ep && ep->ydt == QL_DT_BF16 ? 2 : 4))))
        return QL_ERR_ALIGN;
    if (M == 0)
        return QL_OK;
    const Mx4Args t{qx, sx, (const uint8_t *)codes, scales, (float *)Y, kernel_epilogue(ep),
                    (int)M, (int)N, (int)K};
    if (mx4_takes(t) && mx4_wins(t, current_cus()))
        return mx4_tiles(t, 64) > MAX_WORKGROUPS ? QL_ERR_UNSUPPORTED
                                             : status(launch_qgemm_mx4(t, stream));
    if (rows_tiles(M, N, false) > MAX_WORKGROUPS)
        return QL_ERR_UNSUPPORTED;
    RowsGroup g{};
    RowsArgs &d = g.d[0];
    d.X = qx;
    d.sx = sx;
    d.codes[0] = (const uint8_t *)codes;
    d.scales[0] = scales;
    d.Y = (float *)Y;
    d.ep = t.ep;
    d.M = (int)M;
    d.N = (int)N;
    d.K = (int)K;
    g.n = 1;
    g.maxM = (int)M;
    return status(launch_qgemm_rows(QL_FMT_MXFP4, false, g, stream));
}

int qlinear_gated_forward(const ql_gated *g, void *H, int hdt, hipStream_t stream)
{
    if (!dt_ok(hdt))
        return QL_ERR_INVALID;
    const int st = check_gated(g);
    if (st != QL_OK)
        return st;
    if (g->M == 0)
        return QL_OK;
    const bool bf = hdt == QL_DT_BF16;
    if (!H || H == (const void *)g->X)
        return QL_ERR_INVALID;
    if (!aligned(H, bf ? 2 : 4))
        return QL_ERR_ALIGN;
    GateArgs t = gate_args(*g);
    t.H = H;
    t.hbf16 = bf;
    t.vec = g->N % 4 == 0 && aligned(H, bf ? 8 : 16);
    return launch_gated(*g, t, stream);
}

int qlinear_gated_backward(const ql_gated *g, const ql_gated_grad *d, hipStream_t stream)
{
    const int st = check_gated(g);
    if (st != QL_OK)
        return st;
    if (!d || !dt_ok(d->dhdt) || (d->dX && !dt_ok(d->dxdt)) || !d->dWg != !d->dWu ||
        (d->dWg && !dt_ok(d->dwdt)))
        return QL_ERR_INVALID;
    const int64_t M = g->M, N = g->N, K = g->K;
    if (N % 8)
        return QL_ERR_SHAPE;
    if (M >= I22 || N >= I22 || product_reaches(M, N, I40) || product_reaches(N, K, I40) ||
        product_reaches(M, K, I40))
        return QL_ERR_UNSUPPORTED;
    if (M > 0 && (!d->dH || !d->dG || !d->dU))
        return QL_ERR_INVALID;
    if (!aligned(d->dH, d->dhdt == QL_DT_BF16 ? 2 : 4) || !aligned(d->dG, 16) ||
        !aligned(d->dU, 16) || !aligned(d->dX, 16) || !aligned(d->dWg, 16) ||
        !aligned(d->dWu, 16) || !aligned(d->dbg, 4) || !aligned(d->dbu, 4))
        return QL_ERR_ALIGN;
    // (M == 0: what it writes of them and reads)
    const void *const outs[] = {d->dWg, d->dWu, d->dbg, d->dbu, d->dG, d->dU, d->dX};
    const void *const ins[] = {g->gate_codes, g->gate_scales, g->up_codes, g->up_scales,
                               g->gate_bias, g->up_bias, d->dH, g->X};
    for (int i = 0; i < (M > 0 ? 7 : 4); ++i) {
        if (outs[i] && (std::find(outs, outs + i, outs[i]) != outs + i ||
                        std::find(ins, ins + (M > 0 ? 8 : 6), outs[i]) != ins + (M > 0 ? 8 : 6)))
            return QL_ERR_INVALID;
    }
    const int cus = current_cus();
    const bool want_x = d->dX && M > 0;
    // workspace: both weights in bf16 (q4, int8: two planes each) where dX is not formed
    // from the compressed ones, then the larger of the products' partial sums (the
    // products run one after the other)
    const int planes = g->fmt == QL_FMT_MXFP4 ? 1 : 2;
    const GradPlan plan = grad_plan(g->fmt, M, N, K, g->gate_scales, g->up_scales, want_x,
                                    d->dWg != nullptr, cus);
    const bool direct = plan.direct;
    const int px = plan.xparts, xrows = plan.xrows, pw = plan.wparts, wrows = plan.wrows;
    const size_t plane = want_x && !direct ? round256((size_t)N * K * 2) : 0;
    const size_t wbytes = 2 * planes * plane;
    const size_t part_bytes = std::max(px > 1 ? (size_t)px * M * K * 4 : 0,
                                       pw > 1 ? (size_t)pw * 2 * N * K * 4 : 0);
    if ((want_x && gemm_tiles(xrows, M, K) * px > MAX_WORKGROUPS) ||
        (d->dWg && gemm_tiles(wrows, N, K) * 2 * pw > MAX_WORKGROUPS))
        return QL_ERR_UNSUPPORTED;
    uint8_t *ws = nullptr;
    bool own = false;
    std::unique_lock<std::mutex> turn;
    if (wbytes + part_bytes && !stream_workspace(wbytes + part_bytes, stream, &ws, &own, &turn))
        return QL_ERR_HIP;
    float *const part = reinterpret_cast<float *>(ws + wbytes);

    int s = QL_OK;
    if (M > 0) {
        GateArgs t = gate_args(*g);
        t.dH = d->dH;
        t.dhbf16 = d->dhdt == QL_DT_BF16;
        t.dG = d->dG;
        t.dU = d->dU;
        t.vec = aligned(d->dH, t.dhbf16 ? 8 : 16);
        s = launch_gated(*g, t, stream);
    }
    auto sum = [&](int problems, int p, int64_t R, int64_t S, void *const *out, int bf16) {
        SplitSum sums[2];
        for (int i = 0; i < problems; ++i) {
            sums[i] = SplitSum{part + (int64_t)i * p * R * S, p, R, S, (float *)out[i],
                               kernel_epilogue(nullptr)};
            sums[i].ep.ybf16 = bf16;
        }
        return status(launch_split_sum(sums, problems, stream));
    };
    if (want_x && direct && s == QL_OK) {
        const DxArgs a{{d->dG, d->dU},
                       {(const uint8_t *)g->gate_codes, (const uint8_t *)g->up_codes},
                       {g->gate_scales, g->up_scales},
                       (int)M, (int)N, (int)K, px, part, d->dX, d->dxdt == QL_DT_BF16, xrows};
        s = status(launch_gemm_dx(g->fmt, a, stream));
        void *const out[1] = {d->dX};
        if (s == QL_OK && px > 1)
            s = sum(1, px, M, K, out, a.outbf16);
    }
    if (want_x && !direct && s == QL_OK) {
        GemmArgs a{};
        for (int i = 0; i < 2; ++i)
            for (int q = 0; q < planes; ++q) {
                a.A[i * planes + q] = i ? d->dU : d->dG;
                a.B[i * planes + q] = (uint16_t *)(ws + (i * planes + q) * plane);
            }
        a.lda = N;
        a.ldb = K;
        a.R = (int)M;
        a.S = (int)K;
        a.C = (int)N;
        a.segs = 2 * planes;
        a.parts = px;
        a.rows = xrows;
        a.part = part;
        a.out[0] = d->dX;
        a.outbf16 = d->dxdt == QL_DT_BF16;
        const DequantJob jobs[2] = {
            {g->gate_codes, g->gate_scales, (void *)a.B[0], planes == 2 ? (void *)a.B[1] : nullptr},
            {g->up_codes, g->up_scales, (void *)a.B[planes],
             planes == 2 ? (void *)a.B[3] : nullptr}};
        if (s == QL_OK)
            s = status(launch_dequantize(g->fmt, jobs, 2, N, K, true, stream));
        if (s == QL_OK)
            s = status(launch_gemm_bf16(false, a, 1, stream));
        if (s == QL_OK && px > 1)
            s = sum(1, px, M, K, a.out, a.outbf16);
    }
    if (d->dWg && s == QL_OK) {
        GemmArgs a{};
        a.A[0] = d->dG;
        a.A[1] = d->dU;
        a.B[0] = g->X;
        a.lda = N;
        a.ldb = K;
        a.R = (int)N;
        a.S = (int)K;
        a.C = (int)M;
        a.segs = 1;
        a.parts = pw;
        a.rows = wrows;
        a.part = part;
        a.out[0] = d->dWg;
        a.out[1] = d->dWu;
        a.outbf16 = d->dwdt == QL_DT_BF16;
        s = status(launch_gemm_bf16(true, a, 2, stream));
        if (s == QL_OK && pw > 1)
            s = sum(2, pw, N, K, a.out, a.outbf16);
    }
    if ((d->dbg || d->dbu) && s == QL_OK)
        s = status(launch_column_sums(d->dG, d->dU, d->dbg, d->dbu, (int)M, (int)N, stream));
    if (own && hipFreeAsync(ws, stream) != hipSuccess)
        return QL_ERR_HIP;
    return s;
}

int qlinear_rotary(const void *x, int64_t ldx, void *o, int64_t ldo, int dt, int64_t rows,
                   int64_t heads, int64_t dh, int64_t rot, const double *freqs,
                   const int64_t *positions, int64_t start, int64_t period, float mscale,
                   int interleaved, int adjoint, hipStream_t stream)
{
    if (!dt_ok(dt))
        return QL_ERR_INVALID;
    if (rows < 0 || heads <= 0 || dh <= 0 || rot < 2 || rot > dh || rot % 2)
        return QL_ERR_SHAPE;
    if (rows > MAX_WORKGROUPS || ldx >= I31 || ldo >= I31 || heads >= I31 || dh >= I31)
        return QL_ERR_UNSUPPORTED;
    if (ldx < heads * dh || ldo < heads * dh || (!positions && period <= 0))
        return QL_ERR_SHAPE;
    if (rows == 0)
        return QL_OK;
    const uintptr_t size = dt == QL_DT_BF16 ? 2 : 4;
    if (!x || !o || !freqs)
        return QL_ERR_INVALID;
    if (!aligned(x, size) || !aligned(o, size) || !aligned(freqs, 8) || !aligned(positions, 8))
        return QL_ERR_ALIGN;
    if (rows_overlap(x, ldx, o, ldo, rows, heads * dh, size))
        return QL_ERR_INVALID;
    RotaryArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.o = o;
    a.ldo = ldo;
    a.rows = rows;
    a.heads = (int)heads;
    a.dh = (int)dh;
    a.rot = (int)rot;
    a.freqs = freqs;
    a.positions = positions;
    a.start = start;
    a.period = positions ? 1 : period;
    a.mscale = mscale;
    a.bf16 = dt == QL_DT_BF16;
    a.interleaved = interleaved != 0;
    a.adjoint = adjoint != 0;
    a.copy = x != o;
    return status(launch_rotary(a, current_cus(), stream));
}

}  // extern "C"
