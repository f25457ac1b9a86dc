"""The normalisation at the ends of fp32: rows of any size without eps, backward
(train_ref.py derives the tolerances)."""
import numpy as np
import pytest

import train_ref as R
from test_gpu_norm import host, within

pytestmark = pytest.mark.gpu

EPS = 1e-6
# one for each number of wavefronts and column groups a row
COLUMNS = [96, 600, 1500, 3000, 5000, 9000]


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def put(torch, x, dtype=None):
    """x in fp32, rounded to dtype, on the GPU, and what it holds in 64 bits.  (Made on the
    host: the values may be subnormal.)"""
    t = torch.from_numpy(np.asarray(x, np.float32))
    t = t if dtype is None else t.to(dtype)
    return t.cuda(), t.double().numpy()


@pytest.mark.parametrize("N", COLUMNS)
@pytest.mark.parametrize("size", [-146, -140, -127, -100, 100, 125])
def test_backward_of_any_size(gpu, N, size):
    """Rows of 2^size, from a few subnormal steps to the largest numbers, eps = 0: u = h rstd,
    and with it dw, are of size 1 whatever rstd is; dx = rstd (...) with dy of rstd's inverse
    size is too.  (dy as small as 2^-120: values of its size may be subnormal, where a rounding
    is off by up to 2^-150 and no part of the value.  Four are rounded before the product
    with rstd: g = dy w, k = mean(g u), which counts |u| times, u k, and g - u k.)"""
    torch, ql = gpu
    rng = np.random.default_rng(abs(N + size))
    M = 7
    for hd in (torch.float32, torch.bfloat16):
        if hd == torch.bfloat16 and size < -130:  # (below its smallest steps)
            continue
        x = rng.uniform(1.0, 4.0, (M, N)) * rng.choice([-1, 1], (M, N))
        h, hv = put(torch, x * 2.0 ** size, hd)
        w, wv = put(torch, 1 + 0.3 * rng.standard_normal(N))
        dy, dyv = put(torch, rng.standard_normal((M, N)))
        _, dw = ql.rms_norm_backward(dy, h, w, 0.0)
        _, want, _, bound = R.norm_grads(dyv, hv, wv, 0.0, 0.0)
        within(host(dw), want, bound)
        dy, dyv = put(torch, rng.standard_normal((M, N)) * 2.0 ** max(size, -120))
        dres, dresv = put(torch, rng.standard_normal((M, N)))
        dx, _ = ql.rms_norm_backward(dy, h, w, 0.0, dres=dres)
        want, _, bound, _ = R.norm_grads(dyv, hv, wv, 0.0, dresv)
        r = 1 / np.sqrt((hv * hv).mean(axis=1, keepdims=True))
        within(host(dx), want, bound + 2.0 ** -150 * r * (3 + np.abs(hv * r)))


@pytest.mark.parametrize("N", [96, 3000, 9000])
def test_backward_of_mixed_sizes(gpu, N):
    """Rows of unlike sizes beside each other: each row's part of dw counts alike."""
    torch, ql = gpu
    rng = np.random.default_rng(N)
    M = 40
    size = rng.integers(-140, 120, (M, 1)).astype(np.float64)
    h, hv = put(torch, rng.uniform(1.0, 4.0, (M, N)) * rng.choice([-1, 1], (M, N)) * 2.0 ** size)
    dy, dyv = put(torch, rng.standard_normal((M, N)))
    dx, dw = ql.rms_norm_backward(dy, h, eps=0.0)
    wx, ww, ex, ew = R.norm_grads(dyv, hv, 1.0, 0.0, 0.0)
    within(host(dw), ww, ew)
    held = np.abs(wx) < 3e38  # (others are past fp32's range)
    assert (np.abs(host(dx) - wx) <= ex)[held].all()


def special(torch, N):
    """Rows among which some are zeros, and which."""
    rng = np.random.default_rng(N + 5)
    x = rng.standard_normal((9, N))
    zero = np.array([0, 3, 4, 8])
    x[zero] = 0.0
    x[4, ::2] = -0.0
    return x, zero, np.setdiff1d(np.arange(9), zero), rng


@pytest.mark.parametrize("N", COLUMNS)
def test_zero_rows_without_eps(gpu, N):
    """A row of zeros has no direction: with eps = 0 its y is 0, and it gives dx = dres and
    nothing to dw, which holds the other rows' sums."""
    torch, ql = gpu
    x, zero, others, rng = special(torch, N)
    x, xv = put(torch, x)
    w, wv = put(torch, 1 + 0.3 * rng.standard_normal(N))
    y, h = ql.rms_norm(x, w, 0.0, residual=torch.zeros_like(x), ydtype=torch.float32)
    assert (y[zero] == 0).all() and (h[zero] == 0).all()
    want = R.norm(xv[others], wv, 0.0)
    within(host(y[others]), want, R.norm_error(want, False))
    if N % 32 == 0:
        qx, sx, _ = ql.rms_norm_int8(x, w, 0.0)
        assert (qx[zero] == 0).all() and (sx[zero] == 0).all()
        alone = ql.rms_norm_int8(x[others].contiguous(), w, 0.0)
        assert torch.equal(qx[others], alone[0]) and torch.equal(sx[others], alone[1])
    dy, dyv = put(torch, rng.standard_normal((9, N)))
    dres, dresv = put(torch, rng.standard_normal((9, N)))
    dx, dw = ql.rms_norm_backward(dy, h, w, 0.0, dres=dres)
    assert torch.equal(dx[zero], dres[zero])
    wx, ww, ex, ew = R.norm_grads(dyv[others], xv[others], wv, 0.0, dresv[others])
    within(host(dx[others]), wx, ex)
    within(host(dw), ww, ew)
    dx, dw = ql.rms_norm_backward(dy, torch.zeros_like(h), w, 0.0)
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("N", [96, 1500, 9000])
def test_backward_keeps_rows_apart(gpu, N):
    """Infinities and NaN in a row of h or dy: the other rows' dx are the same to the bit, and
    dw is not finite only in columns that such a row reaches (an infinite rms makes u 0 but
    at the infinity itself)."""
    torch, ql = gpu
    rng = np.random.default_rng(N)
    h, _ = put(torch, rng.standard_normal((6, N)))
    dy, _ = put(torch, rng.standard_normal((6, N)))
    good = torch.tensor([0, 2, 4, 5], device="cuda")
    want, sums = ql.rms_norm_backward(dy, h, eps=EPS)
    for bad in (float("inf"), float("-inf"), float("nan")):
        for which in (0, 1):
            t = [dy.clone(), h.clone()]
            t[which][1, 7] = t[which][3, 50] = bad
            dx, dw = ql.rms_norm_backward(t[0], t[1], eps=EPS)
            assert torch.equal(dx[good], want[good])
            assert not torch.isfinite(dx[[1, 3]]).all(dim=1).any()
            finite = torch.isfinite(dw)
            assert not finite[[7, 50]].any()
            if which == 1 and bad != bad:
                assert not finite.any()
            else:
                assert finite.sum() == N - 2
