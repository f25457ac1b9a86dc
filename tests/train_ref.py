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
