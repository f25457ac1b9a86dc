"""The normalisation with the residual's addition, and its backward pass, on the GPU
against 64-bit references (train_ref.py derives the tolerances)."""
import numpy as np
import pytest

import train_ref as R

pytestmark = pytest.mark.gpu

EPS = 1e-6
# columns: one, odd, the ends of a wavefront's, a workgroup's and a register group's
# rows, the longest; rows: one, fewer and more than the workgroups that run beside
# each other
SIZES = [(1, 1), (3, 7), (5, 33), (1, 512), (9, 511), (6, 513), (2, 1536), (67, 1000), (4, 2048),
         (3, 2049), (2, 4095), (3, 4104), (2, 8191), (2, 8200), (2, 16384), (1300, 96), (5, 513), (7, 1024), (4, 1025), (1601, 600)]


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def rows(torch, rng, M, N, dtype, pad=0, scale=1.0):
    """A row view [M][N] (pad columns behind each row) and its 64-bit values."""
    t = torch.from_numpy((rng.standard_normal((M, N + pad)) * scale).astype(np.float32))
    t = t.to(dtype).cuda()[:, :N]
    return t, t.double().cpu().numpy()


def host(t):
    return t.double().cpu().numpy()


def dtypes(torch, s):
    return [torch.bfloat16 if c == "b" else torch.float32 for c in s]


def within(got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], bound[bad][:4])


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("types", ["bff", "fbb", "bbb", "fff"])
def test_forward(gpu, M, N, types):
    """y and h of x + residual; views with columns behind each row, whose other
    columns keep what they held."""
    torch, ql = gpu
    xd, rd, yd = dtypes(torch, types)
    rng = np.random.default_rng(M * 31 + N)
    x, _ = rows(torch, rng, M, N, xd, pad=3)
    r, _ = rows(torch, rng, M, N, rd, pad=5, scale=3.0)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(N)).astype(np.float32)).cuda()
    y = torch.full((M, N + 2), 7.0, dtype=yd, device="cuda")
    h = torch.full((M, N + 1), 7.0, dtype=rd, device="cuda")
    got = ql.rms_norm(x, w, EPS, residual=r, h=h[:, :N], y=y[:, :N])
    assert got[0].data_ptr() == y.data_ptr() and got[1].data_ptr() == h.data_ptr()
    v = x.float() + r.float()
    assert torch.equal(h[:, :N], v.to(rd))
    want = R.norm(host(v), host(w), EPS)
    within(host(y[:, :N]), want, R.norm_error(want, yd == torch.bfloat16))
    assert (y[:, N:] == 7).all() and (h[:, N:] == 7).all()


@pytest.mark.parametrize("M,N", [(1, 1), (5, 100), (3, 1536), (2, 5000)])
def test_forward_alone(gpu, M, N):
    """Without a residual and a weight; h on request; in place."""
    torch, ql = gpu
    rng = np.random.default_rng(N)
    x, xv = rows(torch, rng, M, N, torch.float32)
    y, h = ql.rms_norm(x, eps=EPS, ydtype=torch.float32)
    assert h is None
    want = R.norm(xv, 1.0, EPS)
    within(host(y), want, R.norm_error(want, False))
    h = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    y2, h2 = ql.rms_norm(x, eps=EPS, h=h, ydtype=torch.float32)
    assert torch.equal(y, y2) and h2 is h and torch.equal(h, x.to(torch.bfloat16))
    # y in x's place, h in the residual's
    r, _ = rows(torch, rng, M, N, torch.float32)
    want_y, want_h = ql.rms_norm(x, eps=EPS, residual=r, ydtype=torch.float32)
    got_y, got_h = ql.rms_norm(x, eps=EPS, residual=r, h=r, y=x)
    assert got_y is x and got_h is r
    assert torch.equal(got_y, want_y) and torch.equal(got_h, want_h)


@pytest.mark.parametrize("M,N", [(1, 32), (7, 512), (9, 544), (5, 1536), (3, 4096), (3, 8192),
                                 (2, 16384)])
@pytest.mark.parametrize("types", ["bf", "fb"])
def test_int8(gpu, M, N, types):
    """Codes and scales are quantize_act's of the fp32 output, bit for bit, and so
    what forward_w8a8 reads."""
    torch, ql = gpu
    xd, rd = dtypes(torch, types)
    rng = np.random.default_rng(N + M)
    x, _ = rows(torch, rng, M, N, xd)
    r, _ = rows(torch, rng, M, N, rd)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(N)).astype(np.float32)).cuda()
    y, h = ql.rms_norm(x, w, EPS, residual=r, ydtype=torch.float32)
    qx, sx, h8 = ql.rms_norm_int8(x, w, EPS, residual=r)
    want_q, want_s = ql.quantize_act(y)
    assert torch.equal(qx, want_q) and torch.equal(sx, want_s) and torch.equal(h, h8)
    # and by the rule itself
    yv = host(y)
    s = (np.abs(yv).max(axis=1) / 127).astype(np.float16)
    assert np.array_equal(s, sx.view(torch.float16).cpu().numpy())
    q = np.clip(np.rint(yv / s.astype(np.float64)[:, None]), -127, 127)
    assert np.array_equal(q, qx.cpu().numpy())


def test_special_rows(gpu):
    """Rows of zeros, of the smallest and largest values, of infinities and NaN: a row
    keeps to itself."""
    torch, ql = gpu
    N = 640
    x = torch.randn((8, N), device="cuda")
    x[1] = 0.0
    x[2] *= 1e-30
    x[3] *= 1e30
    x[4, 17] = float("inf")
    x[5, 300] = float("nan")
    x[6] = 3.0e38
    v = host(x)
    y = ql.rms_norm(x, eps=EPS, ydtype=torch.float32)[0]
    for i in (0, 1, 2, 3, 6, 7):
        want = R.norm(v[i:i + 1], 1.0, EPS)
        within(host(y[i:i + 1]), want, R.norm_error(want, False))
    # (values over an infinite root are 0, infinity over infinity is none)
    assert torch.isnan(y[4, 17]) and (torch.cat((y[4, :17], y[4, 18:])) == 0).all()
    assert torch.isnan(y[5]).all()
    qx, sx, _ = ql.rms_norm_int8(x, eps=EPS)
    s = sx.view(torch.float16)
    assert torch.isnan(s[4:6]).all() and (qx[4:6] == 0).all()
    assert s[1] == 0 and (qx[1] == 0).all() and torch.isfinite(s[[0, 1, 2, 3, 6, 7]]).all()
    # eps = 0: a row's size does not matter
    y0 = ql.rms_norm(x, eps=0.0, ydtype=torch.float32)[0]
    for i in (2, 3):
        want = R.norm(v[i:i + 1], 1.0, 0.0)
        within(host(y0[i:i + 1]), want, R.norm_error(want, False))


@pytest.mark.parametrize("M,N", SIZES + [(600, 1024), (2100, 40)])
@pytest.mark.parametrize("types", ["bff", "fbb", "bbf", "ffb"])
def test_backward(gpu, M, N, types):
    torch, ql = gpu
    yd, hd, xd = dtypes(torch, types)
    rng = np.random.default_rng(M * 7 + N)
    dy, dyv = rows(torch, rng, M, N, yd, pad=1)
    h, hv = rows(torch, rng, M, N, hd, pad=3, scale=2.0)
    dres, dresv = rows(torch, rng, M, N, xd, pad=2)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(N)).astype(np.float32)).cuda()
    out = torch.full((M, N + 4), 7.0, dtype=xd, device="cuda")
    dx, dw = ql.rms_norm_backward(dy, h, w, EPS, dres=dres, dx=out[:, :N])
    want_x, want_w, ex, ew = R.norm_grads(dyv, hv, host(w), EPS, dresv)
    if xd == torch.bfloat16:
        ex = ex + R.BF16 * (np.abs(want_x) + ex)
    within(host(dx), want_x, ex)
    within(host(dw), want_w, ew)
    assert (out[:, N:] == 7).all()
    again = ql.rms_norm_backward(dy, h, w, EPS, dres=dres, dtype=xd)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    assert ql.rms_norm_backward(dy, h, w, EPS, dres=dres, dtype=xd, weight_grad=False)[1] is None


def test_backward_alone(gpu):
    """Without a weight, a residual's gradient; in place of each input."""
    torch, ql = gpu
    rng = np.random.default_rng(3)
    dy, dyv = rows(torch, rng, 37, 720, torch.float32)
    h, hv = rows(torch, rng, 37, 720, torch.float32)
    dx, dw = ql.rms_norm_backward(dy, h, eps=EPS)
    want_x, want_w, ex, ew = R.norm_grads(dyv, hv, 1.0, EPS, 0.0)
    within(host(dx), want_x, ex)
    within(host(dw), want_w, ew)
    dres = torch.randn_like(dy)
    want = ql.rms_norm_backward(dy, h, eps=EPS, dres=dres)[0]
    for k in range(3):
        t = [dy.clone(), h.clone(), dres.clone()]
        assert torch.equal(ql.rms_norm_backward(t[0], t[1], eps=EPS, dres=t[2], dx=t[k])[0], want)


def test_backward_against_differences(gpu):
    """Central differences of the 64-bit forward along random directions.  The
    third derivative of y along a unit direction d, for rows of size about 1, is of
    order N^0; with steps of 1e-4 of |h| the differences are off by 1e-8 of sum |dy|
    |d|, and dx by its bound."""
    torch, ql = gpu
    rng = np.random.default_rng(9)
    M, N = 6, 160
    dy, dyv = rows(torch, rng, M, N, torch.float32)
    h, hv = rows(torch, rng, M, N, torch.float32)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(N)).astype(np.float32)).cuda()
    wv = host(w)
    dx, dw = ql.rms_norm_backward(dy, h, w, EPS)
    _, _, ex, ew = R.norm_grads(dyv, hv, wv, EPS, 0.0)
    t = 1e-4
    for k in range(8):
        d = rng.standard_normal((M, N))
        diff = ((dyv * (R.norm(hv + t * d, wv, EPS) - R.norm(hv - t * d, wv, EPS))).sum(axis=1)
                / (2 * t))
        slack = 10 * t * t * (np.abs(dyv) * np.abs(wv)).sum(axis=1) * np.abs(d).max() ** 3
        assert (np.abs((host(dx) * d).sum(axis=1) - diff) <= (ex * np.abs(d)).sum(axis=1) + slack).all()
        e = rng.standard_normal(N)
        diff = (dyv * R.norm(hv, e, EPS)).sum()  # linear in the weight
        assert abs((host(dw) * e).sum() - diff) <= (ew * np.abs(e)).sum() + 1e-12


@pytest.mark.parametrize("N", [96, 600, 1500])
def test_backward_without_eps(gpu, N):
    """eps = 0 and a number of rows that leaves places of the last workgroups empty: what
    is not there adds nothing to dw."""
    torch, ql = gpu
    rng = np.random.default_rng(N)
    for M in (1, 3, 3073):
        dy, dyv = rows(torch, rng, M, N, torch.float32)
        h, hv = rows(torch, rng, M, N, torch.float32)
        dx, dw = ql.rms_norm_backward(dy, h, eps=0.0)
        want_x, want_w, ex, ew = R.norm_grads(dyv, hv, 1.0, 0.0, 0.0)
        within(host(dx), want_x, ex)
        within(host(dw), want_w, ew)


def test_no_rows(gpu):
    torch, ql = gpu
    x = torch.empty((0, 64), device="cuda")
    y, h = ql.rms_norm(x, residual=x)
    assert y.shape == (0, 64) and h.shape == (0, 64)
    dx, dw = ql.rms_norm_backward(x, x)
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_graph(gpu):
    """Captured with its gradient, replayed on other inputs between eager calls."""
    torch, ql = gpu
    M, N = 300, 1024
    x, r, dy = (torch.randn((M, N), device="cuda") for _ in range(3))
    w = torch.rand(N, device="cuda")

    def step():
        y, h = ql.rms_norm(x, w, EPS, residual=r)
        q = ql.rms_norm_int8(x, w, EPS, residual=r)
        return (y, h, *q, *ql.rms_norm_backward(dy, h, w, EPS, dres=r))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = step()
    for k in range(4):
        for t in (x, r, dy):
            t.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        copies = [t.clone() for t in got]
        for a, b in zip(copies, step()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
