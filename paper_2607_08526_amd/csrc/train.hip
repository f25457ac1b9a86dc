// C-ABI entry points of include/qlinear_train.h: argument checks, choice of kernel and
// launches.  Every check happens before anything is enqueued; no entry point throws or
// aborts.
#include <algorithm>

#include "internal.h"
#include "qlinear_train.h"

using namespace qlk;

namespace {

constexpr int64_t I31 = (int64_t)1 << 31;

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

bool dt_ok(int dt) { return dt == QL_DT_F32 || dt == QL_DT_BF16; }

uintptr_t element(int dt) { return dt == QL_DT_BF16 ? 2 : 4; }

int status(hipError_t e) { return e == hipSuccess ? QL_OK : QL_ERR_HIP; }

// rows of w bytes at a stride of ld bytes
struct Rows {
    const void *p;
    int64_t ld, w, rows;
};

Rows rows_of(const void *p, int64_t ld, int dt, int64_t rows, int64_t w)
{
    const int64_t size = (int64_t)element(dt);
    return {p, ld * size, w * size, rows};
}

// the same elements, one by one
bool same_rows(const Rows &a, const Rows &b)
{
    return a.p == b.p && a.w == b.w && a.rows == b.rows && (a.rows == 1 || a.ld == b.ld);
}

// whether any byte is of both (rows at unlike strides whose ranges meet: taken as so)
bool share_bytes(const Rows &a, const Rows &b)
{
    if (!a.p || !b.p || !a.rows || !b.rows)
        return false;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    const Rows &lo = pa <= pb ? a : b, &hi = pa <= pb ? b : a;
    const uintptr_t diff = pa <= pb ? pb - pa : pa - pb;
    if (diff >= (uintptr_t)((lo.rows - 1) * lo.ld + lo.w))
        return false;
    if ((lo.rows == 1 && hi.rows == 1) || lo.ld != hi.ld)
        return true;
    // columns of one buffer: apart in every row, or not
    const int64_t apart = (int64_t)(diff % (uintptr_t)lo.ld);
    return apart < lo.w || apart + hi.w > lo.ld;
}

// (backward: there is work for the keys without queries too)
int check_attn(const ql_attn *a, bool backward)
{
    // (scale log2(e) is finite, and no other than 0 is smaller than seq_attn takes it)
    if (!a || !(a->scale >= 0.0f) || a->scale > 2.3e38f || (a->scale > 0.0f && a->scale < 1e-30f))
        return QL_ERR_INVALID;
    if (a->B < 0 || a->Tq < 0 || a->Tk < 0 || a->H <= 0 || a->Hk <= 0 || a->H % a->Hk ||
        a->q_rows < 0 || a->k_rows < 0)
        return QL_ERR_SHAPE;
    if ((a->dh != 64 && a->dh != 128) || a->B >= I31 || a->Tq >= I31 || a->Tk > I31 / 2 ||
        a->H >= 1 << 16 || a->q_rows >= I31 || a->k_rows >= I31 || a->ldq >= 1 << 24 ||
        a->ldk >= 1 << 24 || a->ldv >= 1 << 24)
        return QL_ERR_UNSUPPORTED;
    const int64_t rows = a->Tq * (a->H / a->Hk);  // of a key head's queries
    // (each factor is below 2^31 and 2^16: no product overflows.  Rows are at most 2^29 then,
    // and keys 2^30: the kernels add them in 32 bits)
    if (a->B * a->H >= I31 || (a->Tq && a->B * a->H >= (I31 + a->Tq - 1) / a->Tq) ||
        (a->Tk && a->B * a->Hk >= (I31 + a->Tk - 1) / a->Tk) ||
        a->B * a->Hk * ((rows + 31) / 32) > MAX_WORKGROUPS)
        return QL_ERR_UNSUPPORTED;
    if (a->ldq < a->H * a->dh || a->ldk < a->Hk * a->dh || a->ldv < a->Hk * a->dh ||
        (!a->q_offsets && a->q_rows < a->B * a->Tq) || (!a->k_offsets && a->k_rows < a->B * a->Tk))
        return QL_ERR_SHAPE;
    if (a->B == 0 || (a->Tq == 0 && !backward))
        return QL_OK;
    const bool keys = a->Tk > 0 && a->k_rows > 0;
    if ((a->Tq > 0 && a->q_rows > 0 && !a->q) || (keys && (!a->k || !a->v)))
        return QL_ERR_INVALID;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || a->ldq % 8 ||
        a->ldk % 8 || a->ldv % 8 || !aligned(a->q_offsets, 8) || !aligned(a->k_offsets, 8) ||
        !aligned(a->q_lens, 8) || !aligned(a->k_lens, 8))
        return QL_ERR_ALIGN;
    return QL_OK;
}

SeqAttn seq_attn(const ql_attn &a)
{
    SeqAttn s{};
    s.q = a.q;
    s.k = a.k;
    s.v = a.v;
    s.ldq = a.ldq;
    s.ldk = a.ldk;
    s.ldv = a.ldv;
    s.qrows = a.q_rows;
    s.krows = a.k_rows;
    s.q_off = a.q_offsets;
    s.k_off = a.k_offsets;
    s.q_len = a.q_lens;
    s.k_len = a.k_lens;
    s.B = (int)a.B;
    s.T = (int)a.Tq;
    s.KT = (int)a.Tk;
    s.H = (int)a.H;
    s.Hk = (int)a.Hk;
    s.dh = (int)a.dh;
    s.causal = a.causal != 0;
    s.cus = current_cus();
    // (scale 0: so small that every power of it is 1; quotients by it stay finite)
    s.c = std::max(a.scale * 1.44269504088896340736f, 1e-30f);
    return s;
}

// the inputs' rows, for the checks of outputs against them
struct AttnRows {
    Rows r[7];
};
AttnRows attn_inputs(const ql_attn &a)
{
    return {{rows_of(a.q, a.ldq, QL_DT_BF16, a.q_rows, a.H * a.dh),
             rows_of(a.k, a.ldk, QL_DT_BF16, a.k_rows, a.Hk * a.dh),
             rows_of(a.v, a.ldv, QL_DT_BF16, a.k_rows, a.Hk * a.dh),
             {a.q_offsets, 8 * (a.B + 1), 8 * (a.B + 1), 1},
             {a.k_offsets, 8 * (a.B + 1), 8 * (a.B + 1), 1},
             {a.q_lens, 8 * a.B, 8 * a.B, 1},
             {a.k_lens, 8 * a.B, 8 * a.B, 1}}};
}

bool meets_inputs(const Rows &out, const ql_attn &a)
{
    const AttnRows in = attn_inputs(a);
    return std::any_of(in.r, in.r + 7, [&](const Rows &r) { return share_bytes(out, r); });
}

}  // namespace

extern "C" {

int qlinear_rms_norm(const ql_norm *n, hipStream_t stream)
{
    if (!n || !dt_ok(n->xdt) || ((n->res || n->h) && !dt_ok(n->rdt)) || (n->y && !dt_ok(n->ydt)) ||
        !n->qx != !n->sx || !(n->eps >= 0.0) || n->eps > 3e38)
        return QL_ERR_INVALID;
    const int64_t M = n->M, N = n->N;
    if (M < 0 || N <= 0 || n->ldx < N || (n->res && n->ldr < N) || (n->h && n->ldh < N) ||
        (n->y && n->ldy < N) || (n->qx && N % QL_BLOCK))
        return QL_ERR_SHAPE;
    if (N > NORM_MAX_N || M > MAX_WORKGROUPS || n->ldx >= I31 || n->ldr >= I31 || n->ldh >= I31 ||
        n->ldy >= I31)
        return QL_ERR_UNSUPPORTED;
    if (M == 0)
        return QL_OK;
    if (!n->x || (!n->h && !n->y && !n->qx))
        return QL_ERR_INVALID;
    if (!aligned(n->x, element(n->xdt)) || (n->res && !aligned(n->res, element(n->rdt))) ||
        (n->h && !aligned(n->h, element(n->rdt))) || (n->y && !aligned(n->y, element(n->ydt))) ||
        !aligned(n->weight, 4) || !aligned(n->qx, 16) || !aligned(n->sx, 2))
        return QL_ERR_ALIGN;
    const Rows ins[] = {rows_of(n->x, n->ldx, n->xdt, M, N), rows_of(n->res, n->ldr, n->rdt, M, N),
                        {n->weight, 4 * N, 4 * N, 1}};
    const Rows outs[] = {rows_of(n->h, n->ldh, n->rdt, M, N), rows_of(n->y, n->ldy, n->ydt, M, N),
                         {n->qx, N, N, M}, {n->sx, 2 * M, 2 * M, 1}};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 3; ++j)
            if (share_bytes(outs[i], ins[j]) && !(i < 2 && j < 2 && same_rows(outs[i], ins[j])))
                return QL_ERR_INVALID;
        for (int j = 0; j < i; ++j)
            if (share_bytes(outs[i], outs[j]))
                return QL_ERR_INVALID;
    }
    NormArgs a{};
    a.x = n->x;
    a.res = n->res;
    a.ldx = n->ldx;
    a.ldr = n->ldr;
    a.M = M;
    a.N = (int)N;
    a.xbf16 = n->xdt == QL_DT_BF16;
    a.hbf16 = n->rdt == QL_DT_BF16;
    a.ybf16 = n->ydt == QL_DT_BF16;
    a.weight = n->weight;
    a.eps = n->eps;
    a.inv_n = 1.0 / (double)N;
    a.h = n->h;
    a.y = n->y;
    a.ldh = n->ldh;
    a.ldy = n->ldy;
    a.qx = n->qx;
    a.sx = n->sx;
    return status(launch_norm(a, stream));
}

int qlinear_rms_norm_backward(const ql_norm_grad *g, hipStream_t stream)
{
    if (!g || !dt_ok(g->dydt) || !dt_ok(g->hdt) || !dt_ok(g->dxdt) || !(g->eps >= 0.0) ||
        g->eps > 3e38)
        return QL_ERR_INVALID;
    const int64_t M = g->M, N = g->N;
    if (M < 0 || N <= 0 || g->lddy < N || g->ldh < N || (g->dres && g->lddres < N) || g->lddx < N)
        return QL_ERR_SHAPE;
    if (N > NORM_MAX_N || M > MAX_WORKGROUPS || g->lddy >= I31 || g->ldh >= I31 ||
        g->lddres >= I31 || g->lddx >= I31)
        return QL_ERR_UNSUPPORTED;
    if (M > 0 && (!g->dy || !g->h || !g->dx))
        return QL_ERR_INVALID;
    if (!aligned(g->dy, element(g->dydt)) || !aligned(g->h, element(g->hdt)) ||
        !aligned(g->dres, element(g->dxdt)) || !aligned(g->dx, element(g->dxdt)) ||
        !aligned(g->weight, 4) || !aligned(g->dw, 4))
        return QL_ERR_ALIGN;
    const Rows ins[] = {rows_of(g->dy, g->lddy, g->dydt, M, N), rows_of(g->h, g->ldh, g->hdt, M, N),
                        rows_of(g->dres, g->lddres, g->dxdt, M, N), {g->weight, 4 * N, 4 * N, 1}};
    const Rows outs[] = {rows_of(g->dx, g->lddx, g->dxdt, M, N), {g->dw, 4 * N, 4 * N, 1}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 4; ++j)
            if (share_bytes(outs[i], ins[j]) && !(i == 0 && j < 3 && same_rows(outs[i], ins[j])))
                return QL_ERR_INVALID;
    if (share_bytes(outs[0], outs[1]))
        return QL_ERR_INVALID;
    if (M == 0 && !g->dw)
        return QL_OK;
    NormGradArgs a{};
    a.dy = g->dy;
    a.h = g->h;
    a.dres = g->dres;
    a.lddy = g->lddy;
    a.ldh = g->ldh;
    a.ldres = g->lddres;
    a.M = M;
    a.N = (int)N;
    a.ybf16 = g->dydt == QL_DT_BF16;
    a.hbf16 = g->hdt == QL_DT_BF16;
    a.dbf16 = g->dxdt == QL_DT_BF16;
    a.weight = g->weight;
    a.eps = g->eps;
    a.inv_n = 1.0 / (double)N;
    a.dx = g->dx;
    a.lddx = g->lddx;
    a.dw = g->dw;
    const int parts = norm_grad_parts(M, a.N, current_cus());
    uint8_t *ws = nullptr;
    bool own = false;
    std::unique_lock<std::mutex> turn;
    if (g->dw && parts && !stream_workspace((size_t)parts * N * 4, stream, &ws, &own, &turn))
        return QL_ERR_HIP;
    a.part = reinterpret_cast<float *>(ws);
    const int s = status(launch_norm_grad(a, parts, stream));
    if (own && hipFreeAsync(ws, stream) != hipSuccess)
        return QL_ERR_HIP;
    return s;
}

int qlinear_attention_forward(const ql_attn *a, void *o, int64_t ldo, int odt, float *lse,
                              hipStream_t stream)
{
    if (!dt_ok(odt))
        return QL_ERR_INVALID;
    const int st = check_attn(a, false);
    if (st != QL_OK)
        return st;
    if (ldo < a->H * a->dh)
        return QL_ERR_SHAPE;
    if (ldo >= I31)
        return QL_ERR_UNSUPPORTED;
    if (a->B == 0 || a->Tq == 0 || a->q_rows == 0)
        return QL_OK;
    if (!o)
        return QL_ERR_INVALID;
    if (!aligned(o, odt == QL_DT_BF16 ? 8 : 16) || ldo % 4 || !aligned(lse, 4))
        return QL_ERR_ALIGN;
    const Rows out = rows_of(o, ldo, odt, a->q_rows, a->H * a->dh);
    const Rows sums = {lse, 4 * a->q_rows, 4 * a->q_rows, a->H};
    if (meets_inputs(out, *a) || meets_inputs(sums, *a) || share_bytes(out, sums))
        return QL_ERR_INVALID;
    SeqAttnOut t{};
    t.s = seq_attn(*a);
    t.o = o;
    t.ldo = ldo;
    t.obf16 = odt == QL_DT_BF16;
    t.lse = lse;
    // (no more workgroups than MAX_WORKGROUPS: check_attn bounds those of 32 rows, the fewest
    // of any form, and forms in parts have few)
    const SeqAttnPlan plan = seq_attn_plan(t.s);
    t.splits = plan.splits;
    uint8_t *ws = nullptr;
    bool own = false;
    std::unique_lock<std::mutex> turn;
    const size_t bytes = seq_attn_bytes(t.s, plan);
    if (bytes && !stream_workspace(bytes, stream, &ws, &own, &turn))
        return QL_ERR_HIP;
    t.part = reinterpret_cast<float *>(ws);
    const int s = status(launch_seq_attn(t, plan, stream));
    if (own && hipFreeAsync(ws, stream) != hipSuccess)
        return QL_ERR_HIP;
    return s;
}

int qlinear_attention_backward(const ql_attn *a, const ql_attn_grad *g, hipStream_t stream)
{
    const int st = check_attn(a, true);
    if (st != QL_OK)
        return st;
    if (!g || !dt_ok(g->odt) || !dt_ok(g->dt) || !g->dk != !g->dv)
        return QL_ERR_INVALID;
    const int64_t wide = a->H * a->dh, narrow = a->Hk * a->dh;
    if (g->ldo < wide || g->lddo < wide || g->lddq < wide ||
        (g->dk && (g->lddk < narrow || g->lddv < narrow)))
        return QL_ERR_SHAPE;
    if (g->ldo >= I31 || g->lddo >= 1 << 24 || g->lddq >= I31 || g->lddk >= I31 || g->lddv >= I31)
        return QL_ERR_UNSUPPORTED;
    if (a->B == 0)
        return QL_OK;
    const bool queries = a->Tq > 0 && a->q_rows > 0;
    if (queries && (!g->o || !g->lse || !g->dO || !g->dq))
        return QL_ERR_INVALID;
    const uintptr_t grads = g->dt == QL_DT_BF16 ? 8 : 16;
    if (!aligned(g->o, g->odt == QL_DT_BF16 ? 8 : 16) || g->ldo % 4 || !aligned(g->lse, 4) ||
        !aligned(g->dO, 16) || g->lddo % 8 || !aligned(g->dq, grads) || !aligned(g->dk, grads) ||
        !aligned(g->dv, grads) || g->lddq % 4 || (g->dk && (g->lddk % 4 || g->lddv % 4)))
        return QL_ERR_ALIGN;
    const Rows more[] = {rows_of(g->o, g->ldo, g->odt, a->q_rows, wide),
                         rows_of(g->dO, g->lddo, QL_DT_BF16, a->q_rows, wide),
                         {g->lse, 4 * a->q_rows, 4 * a->q_rows, a->H}};
    const Rows outs[] = {rows_of(g->dq, g->lddq, g->dt, a->q_rows, wide),
                         rows_of(g->dk, g->lddk, g->dt, a->k_rows, narrow),
                         rows_of(g->dv, g->lddv, g->dt, a->k_rows, narrow)};
    for (int i = 0; i < 3; ++i) {
        if (meets_inputs(outs[i], *a))
            return QL_ERR_INVALID;
        for (const Rows &r : more)
            if (share_bytes(outs[i], r))
                return QL_ERR_INVALID;
        for (int j = 0; j < i; ++j)
            if (share_bytes(outs[i], outs[j]))
                return QL_ERR_INVALID;
    }
    SeqAttnGrad t{};
    t.s = seq_attn(*a);
    if (!queries)
        t.s.T = 0;
    t.o = g->o;
    t.ldo = g->ldo;
    t.obf16 = g->odt == QL_DT_BF16;
    t.lse = g->lse;
    t.dO = g->dO;
    t.lddo = g->lddo;
    t.dq = g->dq;
    t.dk = g->dk;
    t.dv = g->dv;
    t.lddq = g->lddq;
    t.lddk = g->lddk;
    t.lddv = g->lddv;
    t.bf16 = g->dt == QL_DT_BF16;
    t.scale = a->scale;
    const SeqAttnGradPlan plan = seq_attn_grad_plan(t.s, t.dk != nullptr);
    if (seq_attn_grad_workgroups(t.s, plan) > MAX_WORKGROUPS)
        return QL_ERR_UNSUPPORTED;
    t.qparts = plan.qparts;
    t.kparts = plan.kparts;
    uint8_t *ws = nullptr;
    bool own = false;
    std::unique_lock<std::mutex> turn;
    const size_t bytes = seq_attn_grad_bytes(t.s, plan);
    if (bytes && !stream_workspace(bytes, stream, &ws, &own, &turn))
        return QL_ERR_HIP;
    t.sums = reinterpret_cast<float *>(ws);
    const int s = status(launch_seq_attn_grad(t, stream));
    if (own && hipFreeAsync(ws, stream) != hipSuccess)
        return QL_ERR_HIP;
    return s;
}

}  // extern "C"
