"""64-bit references of the operators of include/qlinear_train.h, in numpy and
written from their formulas, and the tolerances that their arithmetic allows.
"""
import numpy as np

BF16, F32 = 2.0 ** -8, 2.0 ** -24  # half a step of a rounding, relative


def half_step(bf16):
    return BF16 if bf16 else F32


# ---- normalisation -----------------------------------------------------------

def norm(v, w, eps):
    """y of the rows v (64-bit values of fp32 numbers; w may be 1)."""
    return v * w / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)


def norm_error(y, bf16):
    """fp64 to the last step, one rounding to fp32, for bf16 one more."""
    return np.abs(y) * (1.001 * F32 + (BF16 if bf16 else 0.0)) + 2.0 ** -149


def norm_grads(dy, h, w, eps, dres):
    """dx, dw and the bounds of their fp32 arithmetic, before dx's own rounding.

    The kernel has r and k = r mean(g u) from fp64 sums, rounded once; u = h r and g =
    dy w take a rounding each, and so do u k, the difference and the sum with dres: g r
    is off by 2 steps, u k by 4 (r, u, k, the product), of the size of each.  dw: u is
    off by 2 steps, and M additions in any order by M of the sum of magnitudes."""
    M, N = h.shape
    r = 1 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    u, g = h * r, dy * w
    k = r * (g * u).mean(axis=1, keepdims=True)
    own = g * r - u * k
    dx = dres + own
    ex = F32 * (2 * np.abs(g * r) + 4 * np.abs(u * k) + np.abs(own) + np.abs(dx)) * 1.001
    ex += N * 2.0 ** -52 * np.abs(u) * r * np.abs(g * u).mean(axis=1, keepdims=True) + 2.0 ** -140
    dw = (dy * u).sum(axis=0)
    ew = (M + 3) * F32 * np.abs(dy * u).sum(axis=0) + 2.0 ** -140
    return dx, dw, ex, ew


# ---- masked attention --------------------------------------------------------

STEP = 2.0 ** -23  # a rounding of an accumulation, whichever way the matrix cores round


class Seq:
    """Rows of one sequence on both sides: first row, live rows, rows of its place."""

    def __init__(self, q, k):
        (self.q, self.n, self.qcap), (self.k, self.m, self.kcap) = q, k


def heads(x, first, n, H, dh):
    """[H][n][dh] of n rows."""
    return x[first: first + n, : H * dh].reshape(n, H, dh).transpose(1, 0, 2)


def attention(q, k, v, seqs, H, Hk, dh, scale, causal, out_bf16, dO=None, grad_bf16=True):
    """O, lse (and dq, dk, dv) of the 64-bit values of bf16 rows, each with the bound of
    its error: a dict of (value, bound); rows of no sequence NaN.

    With F = 2^-24 and a score's sum off by e = dh STEP sum |q k| scale, and by 4 F (|s| +
    |max|) from its scaling and the difference of rounded products, a probability is off
    by x = e + 4 F (|s| + |max|) + 2^-21 of itself (2^-21: the exponential's last steps).
    The running maximum may trail by 8 powers of two: no more roundings by that than
    one a tile, counted with the sums' (n + 64 for n keys).
      lse: x, the sum's m F, the logarithm's and the last products' 8 F (|lse| + |max| + 1).
      O: sum P |V| times (bf16 of P, 2 x, the sum's (m + 64) STEP), and its rounding.
    Backward, with d = sum dO O: the P of the backward pass comes from lse, off by x + e(lse);
    dP by dh STEP sum |dO V|; d by what O is off by (times |dO|, as the O given is the
    rounded one) and dh STEP sum |dO O|.  dS = P (dP - d) is rounded to bf16 as P is, and the sums
    over n rows take n STEP; dq and dk carry the factor scale, two roundings."""
    F = F32
    out = {"O": np.full((q.shape[0], H * dh), np.nan),
           "lse": np.full((H, q.shape[0]), np.nan)}
    if dO is not None:
        out |= {"dq": np.full((q.shape[0], H * dh), np.nan),
                "dk": np.full((k.shape[0], Hk * dh), np.nan),
                "dv": np.full((k.shape[0], Hk * dh), np.nan)}
    err = {name: np.zeros_like(x) for name, x in out.items()}
    rnd = lambda x, e, bf16: e + half_step(bf16) * (np.abs(x) + e) + 2.0 ** -133

    def put(name, first, cap, n, val, e, bf16):
        """[H][n][dh] into rows, zeros up to cap."""
        for a, x in ((out[name], val), (err[name], rnd(val, e, bf16))):
            a[first: first + cap] = 0.0
            a[first: first + n] = x.transpose(1, 0, 2).reshape(n, a.shape[1])

    for s in seqs:
        n, m, G = s.n, s.m, H // Hk
        Q = heads(q, s.q, n, H, dh)
        K, V = (np.repeat(heads(x, s.k, m, Hk, dh), G, axis=0) for x in (k, v))
        see = np.ones((n, m), bool)
        if causal:
            see = np.arange(m)[None, :] <= np.arange(n)[:, None] + m - n
        T = lambda x: x.transpose(0, 2, 1)
        S = np.where(see, Q @ T(K) * scale, -np.inf)
        e = dh * STEP * (np.abs(Q) @ T(np.abs(K))) * scale
        some = see.any(axis=1)[None, :, None] & np.ones((H, n, 1), bool)
        top = np.where(some, S.max(axis=2, keepdims=True, initial=-np.inf), 0.0)
        P = np.where(see, np.exp(np.where(see, S, 0.0) - top), 0.0)
        total = P.sum(axis=2, keepdims=True)
        P = P / np.where(some, total, 1.0)
        with np.errstate(divide="ignore"):
            lse = np.where(some, top + np.log(total), -np.inf)
        x = np.where(see, e + 4 * F * (np.abs(np.where(see, S, 0.0)) + np.abs(top)) + 2.0 ** -21, 0.0)
        xm = x.max(axis=2, keepdims=True, initial=0.0)
        el = np.where(some, xm + (m + 64) * F + 8 * F * (np.abs(np.where(some, lse, 0.0))
                                                         + np.abs(top) + 1), 0.0)
        O = P @ V
        eO = (P * (BF16 + 2 * xm + 2 * (m + 64) * STEP)) @ np.abs(V)
        put("O", s.q, s.qcap, n, O, eO, out_bf16)
        for a, val in ((out["lse"], lse), (err["lse"], el)):
            a[:, s.q: s.q + s.qcap] = -np.inf if a is out["lse"] else 0.0
            a[:, s.q: s.q + n] = val[:, :, 0]
        if dO is None:
            continue
        D = heads(dO, s.q, n, H, dh)
        dP = D @ T(V)
        d = (D * O).sum(axis=2, keepdims=True)
        eP = P * (x + el + 4 * F * np.abs(np.where(some, lse, 0.0)))
        edP = dh * STEP * (np.abs(D) @ T(np.abs(V)))
        ed = (np.abs(D) * (rnd(O, eO, out_bf16) + dh * STEP * np.abs(O))).sum(axis=2, keepdims=True)
        dS = P * (dP - d)
        edS = eP * (np.abs(dP - d) + edP + ed) + P * (edP + ed + 2 * F * np.abs(dP - d))
        edS = edS + BF16 * (np.abs(dS) + edS)
        eP = eP + BF16 * (P + eP)
        group = lambda y: y.reshape(Hk, G, m, dh).sum(axis=1)
        sums = lambda a, ea, b, c: (ea + (c + 16) * STEP * (a + ea)) @ np.abs(b)
        dq, edq = scale * (dS @ K), scale * sums(np.abs(dS), edS, K, m)
        put("dq", s.q, s.qcap, n, dq, edq + 4 * F * np.abs(dq), grad_bf16)
        dk = scale * group(T(dS) @ Q)
        edk = scale * group(sums(T(np.abs(dS)), T(edS), Q, n * G))
        put("dk", s.k, s.kcap, m, dk, edk + 4 * F * np.abs(dk), grad_bf16)
        dv, edv = group(T(P) @ D), group(sums(T(P), T(eP), D, n * G))
        put("dv", s.k, s.kcap, m, dv, edv, grad_bf16)
    return {name: (out[name], err[name]) for name in out}
