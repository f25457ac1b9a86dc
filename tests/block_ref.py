"""64-bit references of the operators of include/qlinear_block.h, in numpy and
written from their formulas, and the tolerances that their arithmetic allows.

Accumulation: any order of adding K products in fp32 is off by at most K
rounding steps of the sum of magnitudes S = sum |x w|; a step is 2^-23 of it at
most (2^-24 where the matrix cores round to nearest).
"""
import numpy as np
from scipy.special import erf

BLOCK = 32
MAGS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
BF16, F32 = 2.0 ** -8, 2.0 ** -24  # half a step of a rounding, relative
STEP = 2.0 ** -23
PLANES = 2.0 ** -18                # a weight as the sum of two bf16


def mx_encode(x):
    """(codes 0..15 [R][K], scale bytes [R][K/32]) of finite x, by comparing each
    value with every magnitude (ties to the even code)."""
    R, K = x.shape
    b = x.astype(np.float64).reshape(R, -1, BLOCK)
    top = np.abs(b).max(axis=2)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
    e = np.clip(e, -127, 127)
    v = np.abs(b) / np.ldexp(1.0, e)[:, :, None]
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])  # even codes first: they win ties
    d = np.abs(v[..., None] - MAGS[order])
    code = order[np.argmin(d, axis=-1)]
    code = code + 8 * np.signbit(b)
    return code.reshape(R, K).astype(np.uint8), (e + 127).astype(np.uint8)


def pack4(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def mx_decode(codes, scales):
    """Values of unpacked codes and scale bytes (255: NaN)."""
    v = np.where(codes & 8, -MAGS[codes & 7], MAGS[codes & 7])
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(codes.shape[0], -1, BLOCK) * s[:, :, None]).reshape(codes.shape)


def int_encode(x, q):
    """int8 / q4 codes and fp16 scales (the rule of include/qlinear.h, well inside
    its ranges)."""
    b = x.astype(np.float64).reshape(x.shape[0], -1, BLOCK)
    s = (np.abs(b).max(axis=2) / q).astype(np.float16)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s[:, :, None] > 0, np.rint(b / s.astype(np.float64)[:, :, None]), 0)
    return np.clip(c, -q, q).astype(np.int8).reshape(x.shape), s


def int_decode(codes, scales):
    b = codes.astype(np.float64).reshape(codes.shape[0], -1, BLOCK)
    return (b * scales.astype(np.float64)[:, :, None]).reshape(codes.shape)


def weight(fmt, W):
    """(packed codes, scales, 64-bit values) of a weight; fmt "mxfp4", "q4" or
    "int8"."""
    if fmt == "mxfp4":
        c, s = mx_encode(W)
        return pack4(c), s, mx_decode(c, s)
    c, s = int_encode(W, 7 if fmt == "q4" else 127)
    packed = pack4(c.view(np.uint8) & 15) if fmt == "q4" else c.view(np.uint8)
    return packed, s.view(np.int16), int_decode(c, s)


def product(X, W):
    """(X W^T, bound of its accumulation error)."""
    Y = X @ W.T
    return Y, X.shape[1] * STEP * (np.abs(X) @ np.abs(W).T)


def act(kind, g):
    """act, its derivative, and a bound of the second derivative."""
    if kind == "silu":
        s = 1 / (1 + np.exp(-g))
        return g * s, s * (1 + g * (1 - s)), 0.51
    if kind == "gelu":
        P = (1 + erf(g / np.sqrt(2))) / 2
        return g * P, P + g * np.exp(-g * g / 2) / np.sqrt(2 * np.pi), 0.8
    return g, np.ones_like(g), 0.0


def gated(X, Wg, Wu, bg, bu, kind, planes):
    """H, its error bound before the output's rounding, and (G, U, their bounds).
    act' is at most 1.13; the kernels' act is off by 1e-6 of |g| at most (2e-7 from
    the normal distribution's approximation and a few fp32 steps)."""
    G, eG = product(X, Wg)
    U, eU = product(X, Wu)
    if planes:
        eG, eU = eG + PLANES * (np.abs(X) @ np.abs(Wg).T), eU + PLANES * (np.abs(X) @ np.abs(Wu).T)
    G, U = G + bg, U + bu
    eG, eU = eG + 4 * F32 * np.abs(G), eU + 4 * F32 * np.abs(U)
    a, _, _ = act(kind, G)
    ea = 1.13 * eG + 1e-6 * np.abs(G)
    return a * U, ea * (np.abs(U) + eU) + np.abs(a) * eU + 4 * F32 * np.abs(a * U), (G, U, eG, eU)


def gated_grads(dH, G, U, eG, eU, kind):
    """dG, dU and their bounds, the rounding to bf16 in them."""
    a, da, d2 = act(kind, G)
    ea = 1.13 * eG + 1e-6 * np.abs(G)
    eda = d2 * eG + 4e-6 * (1 + np.abs(G))
    dU, dG = dH * a, dH * U * da
    eU_ = np.abs(dH) * ea
    eG_ = np.abs(dH) * (eU * (np.abs(da) + eda) + np.abs(U) * eda)
    rnd = lambda v, e: e + (np.abs(v) + e) * (BF16 + 4 * F32)
    return dG, dU, rnd(dG, eG_), rnd(dU, eU_)


def rotary(x, heads, dh, freqs, positions, interleaved, mscale, adjoint):
    """x [rows][heads * dh] turned, and the error bound in fp32: sine and cosine are
    off by 2^-22 at most, then three roundings."""
    rows, rot = x.shape[0], 2 * len(freqs)
    t = positions.astype(np.float64)[:, None] * freqs[None, :]
    t = np.remainder(t, 2 * np.pi) * (-1 if adjoint else 1)
    c, s = np.cos(t)[:, None, :] * mscale, np.sin(t)[:, None, :] * mscale
    y = x.reshape(rows, heads, dh).copy()
    i = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    j = i + (1 if interleaved else rot // 2)
    a, b = x.reshape(rows, heads, dh)[:, :, i], x.reshape(rows, heads, dh)[:, :, j]
    y[:, :, i], y[:, :, j] = a * c - b * s, b * c + a * s
    e = np.zeros_like(y)
    e[:, :, i] = e[:, :, j] = (np.abs(a) + np.abs(b)) * abs(mscale) * 2.0 ** -21
    return y.reshape(x.shape), e.reshape(x.shape)
