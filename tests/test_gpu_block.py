"""The operators of include/qlinear_block.h, and MXFP4 through the library's
other entry points, against 64-bit references (block_ref.py, where the
tolerances come from)."""
import ctypes

import numpy as np
import pytest

import block_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def fmts(ql):
    return {"mxfp4": ql.FMT_MXFP4, "q4": ql.FMT_Q4, "int8": ql.FMT_INT8}


def acts(ql):
    return {"none": ql.ACT_NONE, "gelu": ql.ACT_GELU, "silu": ql.ACT_SILU}


def dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(torch, a):
    """(device bf16 tensor, its 64-bit values) of a numpy array."""
    t = torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def host(t):
    return t.detach().double().cpu().numpy()


def check(got, want, bound, what):
    got = host(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape, what
    off = np.abs(got - want) - bound
    assert np.all(off <= 0), f"{what}: {np.max(off):.3e} beyond the bound at {np.argmax(off)}"


# ---- MXFP4 -------------------------------------------------------------------

def adversarial(rng, rows, K):
    """Blocks with every tie, saturation, zeros of both signs, subnormals and the
    largest and smallest exponents."""
    x = rng.standard_normal((rows, K)).astype(np.float32)
    b = x.reshape(-1, 32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    for i in range(b.shape[0]):
        k = i % 9
        if k == 1:
            b[i, 0], b[i, 1:8], b[i, 8:15] = 7.9, ties, -ties
        elif k == 2:
            b[i] = 0.0
            b[i, 3] = -0.0
        elif k == 3:
            b[i] *= np.float32(2.0 ** -130)  # subnormal inputs
        elif k == 4:
            b[i] = np.sign(b[i]) * np.float32(3.3e38) * (np.arange(32) % 5 / 4).astype(np.float32)
        elif k == 5:
            e = np.float32(2.0 ** float(rng.integers(-100, 100)))
            b[i, 0], b[i, 1:8] = 4 * e, ties * e
            b[i, 8:15] = np.nextafter(ties, np.float32(9)) * e
            b[i, 15:22] = -np.nextafter(ties, np.float32(0)) * e
        elif k == 6:
            b[i] = np.float32(1.4e-45) * rng.integers(0, 9, 32)
        elif k == 7:
            b[i, 5] = np.float32(np.nextafter(np.float32(8), np.float32(0)))
    return x


@pytest.mark.parametrize("rows,K", [(1, 32), (3, 96), (13, 1536), (200, 1056), (129, 64)])
def test_mx_quantize(gpu, rows, K):
    torch, ql = gpu
    x = adversarial(np.random.default_rng(rows + K), rows, K)
    c, s = R.mx_encode(x)
    for codes, scales in (ql.quantize(ql.FMT_MXFP4, dev(torch, x)),
                          ql.quantize_act_mx(dev(torch, x))):
        np.testing.assert_array_equal(scales.cpu().numpy(), s)
        np.testing.assert_array_equal(codes.cpu().numpy(), R.pack4(c))
        np.testing.assert_array_equal(host(ql.dequantize(ql.FMT_MXFP4, codes, scales)),
                                      R.mx_decode(c, s))
        w = ql.dequantize(ql.FMT_MXFP4, codes, scales, dtype=torch.bfloat16)
        np.testing.assert_array_equal(host(w), R.mx_decode(c, s))
    xb, xv = bf16(torch, x)
    c, s = R.mx_encode(xv)
    codes, scales = ql.quantize_act_mx(xb)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)
    np.testing.assert_array_equal(codes.cpu().numpy(), R.pack4(c))


def test_mx_not_finite(gpu):
    """A weight with a NaN or Inf is refused; an activation block with one becomes
    NaN, the blocks beside it keep their values."""
    torch, ql = gpu
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones((4, 128), np.float32)
        x[2, 70] = bad
        with pytest.raises(ql.QLinearError, match="QL_ERR_RANGE"):
            ql.quantize(ql.FMT_MXFP4, dev(torch, x))
        for t in (dev(torch, x), dev(torch, x).to(torch.bfloat16)):
            codes, scales = ql.quantize_act_mx(t)
            v = host(ql.dequantize(ql.FMT_MXFP4, codes, scales))
            want = np.ones((4, 128))
            want[2, 64:96] = np.nan
            np.testing.assert_array_equal(v, want)
            wc, ws = ql.quantize(ql.FMT_MXFP4, torch.ones((40, 128), device="cuda"))
            Y = host(ql.forward_mx(codes, scales, wc, ws, 40))
            assert np.isnan(Y[2]).all() and (Y[[0, 1, 3]] == 128).all()


@pytest.mark.parametrize("fmt", ["q4", "int8"])
def test_dequantize_int(gpu, fmt):
    torch, ql = gpu
    W = np.random.default_rng(3).standard_normal((37, 160)).astype(np.float32)
    codes, scales = ql.quantize(fmts(ql)[fmt], dev(torch, W))
    c, s, v = R.weight(fmt, W)
    np.testing.assert_array_equal(host(ql.dequantize(fmts(ql)[fmt], codes, scales)), v)
    got = ql.dequantize(fmts(ql)[fmt], codes, scales, dtype=torch.bfloat16)
    check(got, v, np.abs(v) * R.BF16, "bf16")


def test_mx_every_scale(gpu):
    """Every scale byte and code through the products: exact where one product makes
    the output, subnormal and NaN scales among them."""
    torch, ql = gpu
    codes = np.zeros((256, 32), np.uint8)
    codes[:, 0] = np.arange(256) % 16
    scales = np.arange(256, dtype=np.uint8).reshape(256, 1)
    v = R.mx_decode(codes, scales)[:, 0]
    c, s = dev(torch, R.pack4(codes)), dev(torch, scales)
    for x, dt in ((1.0, torch.bfloat16), (0.125, torch.bfloat16), (1.0, torch.float32),
                  (0.125, torch.float32)):
        X = torch.zeros((2, 32), dtype=dt, device="cuda")
        X[:, 0] = x
        Y = host(ql.forward(ql.FMT_MXFP4, X, c, s, 256))
        # (magnitudes from 2^128, with scales that quantization never gives, are no
        # fp32: infinite, and NaN where a zero meets them, as the smaller terms of an
        # fp32 activation do)
        big = np.abs(v) >= 2.0 ** 128
        want = (np.where(big, 0, v) * x).astype(np.float32).astype(np.float64)
        for row in Y:
            np.testing.assert_array_equal(row[~big], want[~big])
            assert not np.isfinite(row[big]).any()
    # 4-bit activations: 1 times every scale
    xc = np.zeros((1, 32), np.uint8)
    xc[0, 0] = 2
    qx = dev(torch, R.pack4(xc))
    for sx in (0, 100, 127, 160, 254, 255):
        Y = host(ql.forward_mx(qx, torch.full((1, 1), sx, dtype=torch.uint8, device="cuda"), c, s,
                               256))[0]
        with np.errstate(over="ignore", invalid="ignore"):
            want = v * (np.nan if sx == 255 else 2.0 ** (sx - 127))
            want = want.astype(np.float32).astype(np.float64)
        np.testing.assert_array_equal(Y, want)


# from one value to the large tiles: reductions of every residue that the kernels
# tell apart (32, 128, 256, 512), widths that end inside a tile or a group of four
SHAPES = [(1, 1, 32), (1, 200, 96), (3, 33, 64), (8, 2000, 128), (16, 1000, 160), (9, 130, 6144),
          (17, 64, 1056), (33, 96, 512), (40, 300, 384), (64, 257, 256), (65, 1024, 128),
          (130, 40, 2048), (130, 640, 2176), (256, 1030, 1024), (300, 520, 384), (513, 768, 1536),
          (520, 2052, 128), (1100, 2064, 640), (1100, 4100, 256), (1100, 4099, 384),
          (1100, 4100, 512), (1030, 4100, 1152), (1030, 4102, 1536), (130, 1000, 416),
          (300, 2050, 1056), (1100, 4100, 224), (1100, 4100, 288), (1030, 4100, 1056),
          (1030, 4098, 864), (1900, 4092, 512), (1900, 4090, 544)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("x", ["bf16", "f32", "mx"])
def test_mx_product(gpu, M, N, K, x):
    torch, ql = gpu
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    W = rng.standard_normal((N, K)).astype(np.float32) * np.float32(0.02)
    codes, scales, Wv = R.weight("mxfp4", W)
    X = rng.standard_normal((M, K)).astype(np.float32)
    X[:, ::37] *= 20
    c, s = dev(torch, codes), dev(torch, scales)
    guard = torch.full((M + 2, N), 77.0, device="cuda")
    Y = guard[:M]
    if x == "f32":
        Xv = X.astype(np.float64)
        ql.forward(ql.FMT_MXFP4, dev(torch, X), c, s, N, Y=Y)
    elif x == "bf16":
        Xb, Xv = bf16(torch, X)
        ql.forward(ql.FMT_MXFP4, Xb, c, s, N, Y=Y)
    else:
        Xb, Xv = bf16(torch, X)
        Xv = R.mx_decode(*R.mx_encode(Xv))
        ql.forward_mx(*ql.quantize_act_mx(Xb), c, s, N, Y=Y)
    want, bound = R.product(Xv, Wv)
    check(Y, want, bound + 2.0 ** -26 * np.abs(want), x)
    rel = np.linalg.norm(host(Y) - want) / np.linalg.norm(want)
    assert rel <= 2.0 ** -22 * np.sqrt(K), rel
    assert (guard[M:] == 77.0).all()


def test_mx_extreme_activations(gpu):
    """fp32 activations near the largest and smallest fp32 meet every plane; an
    infinity or a NaN stays in its row."""
    torch, ql = gpu
    rng = np.random.default_rng(5)
    K, N = 96, 48
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32))
    X = rng.standard_normal((5, K)).astype(np.float32)
    X[0] *= np.float32(1e36)
    X[1] *= np.float32(1e-30)
    X[2, 7] = np.inf
    X[3, 8] = np.nan
    Y = host(ql.forward(ql.FMT_MXFP4, dev(torch, X), dev(torch, codes), dev(torch, scales), N))
    want, bound = R.product(X[[0, 1, 4]].astype(np.float64), Wv)
    check(Y[[0, 1, 4]], want, bound, "finite rows")
    assert not np.isfinite(Y[2]).any() and np.isnan(Y[3]).all()


@pytest.mark.parametrize("M,N,K", [(1, 100, 64), (40, 258, 96), (40, 260, 128), (200, 264, 512),
                                   (700, 512, 256), (1100, 4100, 256), (1100, 4098, 512),
                                   (1900, 4092, 512), (1900, 4090, 544)])
@pytest.mark.parametrize("mx", [False, True])
def test_mx_epilogue(gpu, M, N, K, mx):
    """Bias, GELU, residual, steering, bf16 outputs and copies."""
    torch, ql = gpu
    rng = np.random.default_rng(M + N)
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32) * 0.1)
    Xb, Xv = bf16(torch, rng.standard_normal((M, K)))
    bias = rng.standard_normal(N).astype(np.float32)
    resid = rng.standard_normal((M, N)).astype(np.float32)
    d = rng.standard_normal(N).astype(np.float32)
    strength = torch.tensor([0.5], device="cuda")
    c, s = dev(torch, codes), dev(torch, scales)
    if mx:
        Xv = R.mx_decode(*R.mx_encode(Xv))
        q = ql.quantize_act_mx(Xb)
        call = lambda **kw: ql.forward_mx(*q, c, s, N, **kw)
    else:
        call = lambda **kw: ql.forward_ep(ql.FMT_MXFP4, Xb, c, s, N, **kw)
    P, e = R.product(Xv, Wv)
    e = 1.13 * (e + 4 * R.F32 * (np.abs(P) + np.abs(bias))) + 1e-6 * (np.abs(P) + np.abs(bias))
    copy = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    Y = call(bias=dev(torch, bias), act=ql.ACT_GELU, residual=dev(torch, resid),
             steer=(dev(torch, d), 2.0, strength), ycopy=copy)
    want = R.act("gelu", P + bias)[0] + resid + 1.0 * d
    e32 = e + 8 * R.F32 * (np.abs(want) + np.abs(resid) + np.abs(d))
    check(Y, want, e32, "fp32")
    assert torch.equal(copy, Y.to(torch.bfloat16))
    Y = call(bias=dev(torch, bias), ydtype=torch.bfloat16)
    want = P + bias
    check(Y, want, e + R.BF16 * (np.abs(want) + e), "bf16")
    h = dev(torch, resid)
    call(Y=h, residual=h)
    check(h, P + resid, e + 8 * R.F32 * (np.abs(P) + np.abs(resid)), "in place")


def test_mx_groups(gpu):
    """MXFP4 layers in grouped calls, beside other formats, equal to single calls
    bit for bit; the entry point that allocates nothing too."""
    torch, ql = gpu
    rng = np.random.default_rng(8)
    M, shapes = 21, [(96, 64), (64, 256), (300, 64), (64, 256)]
    fm = [ql.FMT_MXFP4, ql.FMT_MXFP4, ql.FMT_Q4, ql.FMT_MXFP4]
    ents, single = [], []
    for i, ((N, K), f) in enumerate(zip(shapes, fm)):
        codes, scales = ql.quantize(f, dev(torch, rng.standard_normal((N, K)).astype(np.float32)))
        X = dev(torch, rng.standard_normal((M, K)).astype(np.float32))
        X = X if i == 3 else X.to(torch.bfloat16)
        ents.append((f, X, codes, scales, N, torch.empty((M, N), device="cuda"), None,
                     ql.ACT_NONE, None))
        single.append(ql.forward(f, X, codes, scales, N))
    for call in (ql.block_forward_ep, ql.block_forward_ep_noalloc):
        for e in ents:
            e[5].fill_(-1)
        call(ents)
        for e, y in zip(ents, single):
            assert torch.equal(e[5], y)
    ql.block_forward([e[:6] for e in ents])
    for e, y in zip(ents, single):
        assert torch.equal(e[5], y)


def test_mx_groups_of_many_rows(gpu):
    """Layers of different kernels and row counts in one call: one row beside the
    tiles, fp32 layers that share their activations, one whose activations take more
    than a slice of the workspace; each against its own reference, and the entry point
    that allocates nothing the same bit for bit."""
    torch, ql = gpu
    rng = np.random.default_rng(18)
    K = 2048
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((520, K)).astype(np.float32) * 0.05)
    c, s = dev(torch, codes), dev(torch, scales)
    big = rng.standard_normal((10500, K)).astype(np.float32)
    tall, few = big[:300], big[:1]
    resid = dev(torch, rng.standard_normal((10500, 520)).astype(np.float32))
    copy = torch.empty((10500, 520), dtype=torch.bfloat16, device="cuda")
    rows = [0, 127, 128, 4999, 10239, 10240, 10241, 10303, 10304, 10499]
    bigd, talld = dev(torch, big), dev(torch, tall)
    f = lambda X, N, Y, r=None, y=None: (ql.FMT_MXFP4, X, c[:N], s[:N], N, Y, None, ql.ACT_NONE,
                                         r, None, y)
    new = lambda M, N, dt=torch.float32: torch.empty((M, N), dtype=dt, device="cuda")
    ents = [f(bigd, 520, new(10500, 520), resid, copy), f(dev(torch, few), 100, new(1, 100)),
            f(talld, 520, new(300, 520)), f(talld, 516, new(300, 516, torch.bfloat16)),
            f(dev(torch, few).to(torch.bfloat16), 520, new(1, 520)),
            f(dev(torch, tall).to(torch.bfloat16), 520, new(300, 520))]
    ql.block_forward_ep(ents)
    first = [e[5].clone() for e in ents] + [copy.clone()]
    P, e = R.product(big[rows].astype(np.float64), Wv)
    want = P + host(resid[rows])
    check(ents[0][5][rows], want, e + 4 * R.F32 * (np.abs(P) + np.abs(want)), "slices")
    assert torch.equal(copy, ents[0][5].to(torch.bfloat16))
    P, e = R.product(tall.astype(np.float64), Wv)
    check(ents[1][5], P[:1, :100], e[:1, :100], "one row")
    check(ents[2][5], P, e, "fp32")
    check(ents[3][5], P[:, :516], (e + R.BF16 * (np.abs(P) + e))[:, :516], "bf16 output")
    P, e = R.product(bf16(torch, tall)[1], Wv)
    check(ents[4][5], P[:1], e[:1], "one bf16 row")
    check(ents[5][5], P, e, "bf16")
    for t in ents:
        t[5].fill_(-1)
    copy.fill_(-1)
    ql.block_forward_ep_noalloc(ents)
    for a, b in zip(first, [t[5] for t in ents] + [copy]):
        assert torch.equal(a, b)


# reductions beyond the staged kernels' 2^22
@pytest.mark.parametrize("M", [1, 21])
def test_mx_longest_reductions(gpu, M):
    torch, ql = gpu
    rng = np.random.default_rng(M)
    K, N = (1 << 22) + 32, 3
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32) * 0.05)
    c, s = dev(torch, codes), dev(torch, scales)
    X = rng.standard_normal((M, K)).astype(np.float32)
    check(ql.forward(ql.FMT_MXFP4, dev(torch, X), c, s, N),
          *R.product(X.astype(np.float64), Wv), "fp32")
    Xb, Xv = bf16(torch, X)
    check(ql.forward(ql.FMT_MXFP4, Xb, c, s, N), *R.product(Xv, Wv), "bf16")
    q = ql.quantize_act_mx(Xb)
    check(ql.forward_mx(*q, c, s, N), *R.product(host(ql.dequantize(ql.FMT_MXFP4, *q)), Wv), "mx")


def test_mx_scales_at_any_byte(gpu):
    """Scale bytes need no alignment: slices that start at odd addresses (which other
    kernels take, that add in another order)."""
    torch, ql = gpu
    rng = np.random.default_rng(9)
    M, N, K = 70, 130, 512
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32))
    X, Xv = bf16(torch, rng.standard_normal((M, K)))
    c, s = dev(torch, codes), dev(torch, scales)
    qx, sx = ql.quantize_act_mx(X)
    Xq = R.mx_decode(*R.mx_encode(Xv))
    for off in (0, 1, 2, 3, 4):
        def shifted(t):
            v = torch.empty(t.numel() + 4, dtype=torch.uint8, device="cuda")
            v = v[off: off + t.numel()].view(t.shape)
            return v.copy_(t)
        odd = shifted(s)
        check(ql.forward(ql.FMT_MXFP4, X, c, odd, N), *R.product(Xv, Wv), f"bf16 {off}")
        check(ql.forward_mx(qx, shifted(sx), c, odd, N), *R.product(Xq, Wv), f"mx {off}")
        want, e, _ = R.gated(Xv, Wv, Wv, 0, 0, "silu", False)
        H = torch.empty((M, N), device="cuda")
        check(ql.gated_forward(ql.FMT_MXFP4, X, (c, odd), (c, odd), H=H), want, e, f"gated {off}")


# ---- gated feed-forward -----------------------------------------------------------

GATED = [(1, 8, 32), (1, 1000, 96), (5, 17, 64), (16, 130, 1056), (33, 64, 160), (64, 72, 256),
         (65, 500, 128), (129, 264, 512), (260, 128, 1536), (700, 640, 384), (9, 40, 4096),
         (20, 1000, 128), (130, 1032, 384), (260, 2048, 256), (1100, 2056, 256), (1100, 2050, 384),
         (1100, 2056, 512), (1030, 2056, 1152), (130, 1032, 416), (1100, 2056, 224),
         (1100, 2056, 288), (1030, 2056, 1056), (1900, 2042, 1536), (1900, 2040, 1568),
         (7, 72, 2080), (400, 2048, 1024), (260, 136, 16384), (70, 320, 12320),
         (320, 72, 25632), (512, 16380, 544)]


def gated_case(torch, fmt, M, N, K, seed, bias):
    rng = np.random.default_rng(seed)
    gate, up = (R.weight(fmt, rng.standard_normal((N, K)).astype(np.float32) / np.sqrt(K))
                for _ in range(2))
    Xb, Xv = bf16(torch, rng.standard_normal((M, K)))
    b = [rng.standard_normal(N).astype(np.float32) * np.float32(0.3) if bias else np.zeros(N)
         for _ in range(2)]
    db = tuple(dev(torch, v) for v in b) if bias else None
    pair = tuple((dev(torch, w[0]), dev(torch, w[1])) for w in (gate, up))
    return rng, Xb, Xv, pair, (gate[2], up[2]), b, db


@pytest.mark.parametrize("M,N,K", GATED)
@pytest.mark.parametrize("fmt", ["mxfp4", "q4", "int8"])
def test_gated_forward(gpu, fmt, M, N, K):
    torch, ql = gpu
    for kind, bias in (("silu", True), ("gelu", False), ("none", True)):
        _, Xb, Xv, pair, (Wg, Wu), b, db = gated_case(torch, fmt, M, N, K, M + N + K, bias)
        want, e, _ = R.gated(Xv, Wg, Wu, b[0], b[1], kind, fmt != "mxfp4")
        guard = torch.full((M + 1, N), 55.0, device="cuda")
        ql.gated_forward(fmts(ql)[fmt], Xb, *pair, H=guard[:M], bias=db, act=acts(ql)[kind])
        check(guard[:M], want, e, f"{kind} fp32")
        assert (guard[M:] == 55.0).all()
        H = ql.gated_forward(fmts(ql)[fmt], Xb, *pair, bias=db, act=acts(ql)[kind])
        assert H.dtype == torch.bfloat16 and torch.equal(H, guard[:M].to(torch.bfloat16))


@pytest.mark.parametrize("M,N,K", [s for s in GATED if s[1] % 8 == 0])
@pytest.mark.parametrize("fmt", ["mxfp4", "q4", "int8"])
@pytest.mark.parametrize("dhdt", ["f32", "bf16"])
def test_gated_backward(gpu, fmt, M, N, K, dhdt):
    torch, ql = gpu
    kind, bias = ("silu", True) if dhdt == "f32" else ("gelu", False)
    rng, Xb, Xv, pair, (Wg, Wu), b, db = gated_case(torch, fmt, M, N, K, M + N, bias)
    dH = rng.standard_normal((M, N)).astype(np.float32)
    dHd, dHv = bf16(torch, dH) if dhdt == "bf16" else (dev(torch, dH), dH.astype(np.float64))
    for dtype in (torch.float32, torch.bfloat16):
        g = ql.gated_backward(fmts(ql)[fmt], Xb, *pair, dHd, bias=db, act=acts(ql)[kind],
                              weight_grads=True, bias_grads=True, dtype=dtype)
        H, _, (G, U, eG, eU) = R.gated(Xv, Wg, Wu, b[0], b[1], kind, fmt != "mxfp4")
        dG, dU, bG, bU = R.gated_grads(dHv, G, U, eG, eU, kind)
        check(g.gate, dG, bG, "dG")
        check(g.up, dU, bU, "dU")
        # the products, from the bf16 gradients as they were returned
        dGr, dUr = host(g.gate), host(g.up)
        out = lambda v, e: e if dtype == torch.float32 else e + R.BF16 * (np.abs(v) + e)
        dX = dGr @ Wg + dUr @ Wu
        S = np.abs(dGr) @ np.abs(Wg) + np.abs(dUr) @ np.abs(Wu)
        e = S * (2 * N * R.STEP * (1 if fmt == "mxfp4" else 2) +
                 (R.PLANES if fmt != "mxfp4" else 0))
        check(g.X, dX, out(dX, e), "dX")
        for got, d, name in ((g.W_gate, dGr, "dWg"), (g.W_up, dUr, "dWu")):
            dW = d.T @ Xv
            check(got, dW, out(dW, M * R.STEP * (np.abs(d).T @ np.abs(Xv))), name)
        for got, d in ((g.b_gate, dGr), (g.b_up, dUr)):
            check(got, d.sum(axis=0), M * R.STEP * np.abs(d).sum(axis=0), "db")
        # and all of it against the formula in 64 bits
        for got, want in ((g.X, dG @ Wg + dU @ Wu), (g.W_gate, dG.T @ Xv), (g.W_up, dU.T @ Xv)):
            rel = np.linalg.norm(host(got) - want) / max(np.linalg.norm(want), 1e-30)
            assert rel <= 2 * R.BF16, rel


def test_gated_gradient_against_differences(gpu):
    """The gradients against central differences of the 64-bit loss sum(H dH) along
    random directions; the returned ones carry bf16 roundings (2^-8 of each entry,
    so of the norm, twice over)."""
    torch, ql = gpu
    M, N, K = 37, 88, 160
    for fmt, kind in (("mxfp4", "silu"), ("q4", "gelu"), ("int8", "silu")):
        rng, Xb, Xv, pair, W, b, db = gated_case(torch, fmt, M, N, K, 77, True)
        dH = rng.standard_normal((M, N)).astype(np.float32)
        g = ql.gated_backward(fmts(ql)[fmt], Xb, *pair, dev(torch, dH), bias=db,
                              act=acts(ql)[kind], weight_grads=True, bias_grads=True)
        at = [Xv, W[0], W[1], b[0].astype(np.float64), b[1].astype(np.float64)]

        def loss(p):
            return (R.act(kind, p[0] @ p[1].T + p[3])[0] * (p[0] @ p[2].T + p[4]) * dH).sum()

        for i, got in enumerate((g.X, g.W_gate, g.W_up, g.b_gate, g.b_up)):
            v = rng.standard_normal(at[i].shape)
            h = 1e-5
            up, dn = list(at), list(at)
            up[i], dn[i] = at[i] + h * v, at[i] - h * v
            fd = (loss(up) - loss(dn)) / (2 * h)
            d = host(got)
            assert abs((d * v).sum() - fd) <= 4 * R.BF16 * np.linalg.norm(d) * np.linalg.norm(v)


def test_gated_no_rows(gpu):
    """M = 0: nothing to write but the zero gradients of weights and biases."""
    torch, ql = gpu
    _, _, _, pair, _, _, _ = gated_case(torch, "q4", 1, 64, 64, 1, False)
    X = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    assert ql.gated_forward(ql.FMT_Q4, X, *pair).shape == (0, 64)
    g = ql.gated_backward(ql.FMT_Q4, X, *pair, torch.empty((0, 64), device="cuda"),
                          weight_grads=True, bias_grads=True)
    assert g.X.shape == (0, 64) and not g.W_gate.any() and not g.W_up.any()
    assert not g.b_gate.any() and not g.b_up.any()


def test_gated_partial_outputs(gpu):
    """Only the gradients that are asked for, and each the same whatever else is."""
    torch, ql = gpu
    rng, Xb, _, pair, _, _, db = gated_case(torch, "mxfp4", 90, 136, 256, 4, True)
    dH = dev(torch, rng.standard_normal((90, 136)).astype(np.float32))
    call = lambda **kw: ql.gated_backward(ql.FMT_MXFP4, Xb, *pair, dH, bias=db, **kw)
    full = call(weight_grads=True, bias_grads=True)
    none = call(x_grad=False)
    assert none.X is None and none.W_gate is None and none.b_up is None
    assert torch.equal(none.gate, full.gate) and torch.equal(none.up, full.up)
    assert torch.equal(call().X, full.X)
    w = call(x_grad=False, weight_grads=True)
    assert torch.equal(w.W_gate, full.W_gate) and torch.equal(w.W_up, full.W_up)
    b = call(x_grad=False, bias_grads=True)
    assert torch.equal(b.b_gate, full.b_gate) and torch.equal(b.b_up, full.b_up)


# ---- rotary positions ----------------------------------------------------------

ROTARY = [  # rows, heads, dh, rot, extra columns
    (1, 2, 64, 64, 0), (3, 5, 64, 32, 64), (130, 8, 64, 48, 0), (7, 3, 80, 20, 5),
    (2, 1, 6, 2, 1), (65, 48, 64, 64, 1536), (4, 2, 128, 128, 8), (5, 1, 4100, 4100, 0),
    (3000, 4, 64, 16, 0), (9, 160, 128, 128, 8), (1200, 70, 64, 32, 0)]


@pytest.mark.parametrize("rows,heads,dh,rot,extra", ROTARY)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(gpu, rows, heads, dh, rot, extra, dt, interleaved):
    torch, ql = gpu
    rng = np.random.default_rng(rows + heads + rot)
    x = rng.standard_normal((rows, heads * dh + extra)).astype(np.float32)
    t, xv = bf16(torch, x) if dt == "bf16" else (dev(torch, x), x.astype(np.float64))
    pos = rng.integers(-(1 << 20), 1 << 24, rows)
    pos[0] = 0
    freqs, m = ql.rotary_frequencies(rot, scaling="yarn", factor=8.0, context=4096)
    f = freqs.cpu().numpy()
    for adjoint in (False, True):
        want, e = R.rotary(xv[:, :heads * dh], heads, dh, f, pos, interleaved, m, adjoint)
        e = e + (R.BF16 * (np.abs(want) + e) if dt == "bf16" else 0) * (want != xv[:, :heads * dh])
        wide = torch.full((rows + 1, heads * dh + extra + 3), 9.0, dtype=t.dtype, device="cuda")
        out = wide[:rows, :heads * dh]
        kw = dict(dh=dh, positions=dev(torch, pos), interleaved=interleaved, mscale=m,
                  adjoint=adjoint)
        assert ql.rotary(t, heads, freqs, out=out, **kw) is out
        check(out, want, e, "out of place")
        assert (wide[rows:] == 9).all() and (wide[:, heads * dh:] == 9).all()
        inplace = t.clone()
        ql.rotary(inplace, heads, freqs, **kw)
        assert torch.equal(inplace[:, :heads * dh], out)
        assert torch.equal(inplace[:, heads * dh:], t[:, heads * dh:])


def test_rotary_row_positions(gpu):
    """Positions that are not given count up within each sequence; turning back
    (adjoint at mscale 1) gives the input again, to the roundings of both turns."""
    torch, ql = gpu
    B, T, H = 3, 50, 4
    x = torch.randn((B * T, H * 64), device="cuda")
    freqs, _ = ql.rotary_frequencies(64)
    pos = (1000 + torch.arange(T, device="cuda")).repeat(B)
    y = ql.rotary(x, H, freqs, start=1000, T=T, out=torch.empty_like(x))
    assert torch.equal(y, ql.rotary(x, H, freqs, positions=pos, out=torch.empty_like(x)))
    back = ql.rotary(y, H, freqs, start=1000, T=T, adjoint=True)
    assert (back - x).abs().max() <= 2.0 ** -20 * x.abs().max() * 2
    one = ql.rotary(x, H, freqs, out=torch.empty_like(x))
    assert torch.equal(one, ql.rotary(x, H, freqs, positions=torch.arange(B * T, device="cuda"),
                                      out=torch.empty_like(x)))
    assert ql.rotary(x[:0], H, freqs).shape == (0, H * 64)


def test_rotary_overlapping_rows(gpu):
    """Rows that are longer than their distance: only the heads' channels are read
    and written."""
    torch, ql = gpu
    rows, H = 6, 2
    flat = torch.randn(rows * 128 + 64, device="cuda")
    x = flat.as_strided((rows, 192), (128, 1))
    freqs, _ = ql.rotary_frequencies(32)
    want = ql.rotary(flat[:rows * 128].view(rows, 128).clone(), H, freqs)
    out = torch.full((rows, 192), 3.0, device="cuda")
    ql.rotary(x, H, freqs, out=out)
    assert torch.equal(out[:, :128], want) and (out[:, 128:] == 3).all()
    tail = flat[rows * 128:].clone()
    both = torch.cat((flat[:rows * 128].view(rows, 128), torch.empty((rows, 130), device="cuda")),
                     dim=1)
    ql.rotary(both[:, :128], H, freqs, out=both[:, 130:])  # into other columns of the rows
    assert torch.equal(both[:, 130:], want)
    with pytest.raises(ql.QLinearError):
        ql.rotary(both[:, :128], H, freqs, out=both[:, 127:255])
    one = flat[:256].view(1, 256).clone()
    row = ql.rotary(one[:, :128].clone(), H, freqs, start=5)
    ql.rotary(one, H, freqs, start=5, out=one[:, :128])  # one row in place, by another length
    assert torch.equal(one[:, :128], row)
    ql.rotary(x, H, freqs)
    assert torch.equal(flat[:rows * 128].view(rows, 128), want)
    assert torch.equal(flat[rows * 128:], tail)


# ---- offsets past 32 bits ------------------------------------------------------------
# The first 64 rows repeat: whatever lies far must come out as they do, bit for bit
# (the same kernel, and the same order of sums, at another address).

def periodic(torch, t, rows=64):
    """Every row of t equals the row 64 before it."""
    for i in range(rows, t.shape[0], 1 << 13):
        part = t[i: i + (1 << 13)]
        if not torch.equal(part, t[i - rows: i - rows + part.shape[0]]):
            return False
    return True


def test_many_rows_past_32_bits(gpu):
    torch, ql = gpu
    n, g = 2049, torch.Generator(device="cuda").manual_seed(1)
    many = lambda t: t.repeat(n, 1)
    base = torch.randn((64, 32768), generator=g, device="cuda").to(torch.bfloat16)
    X = many(base)
    M = X.shape[0]
    assert X.numel() > 1 << 32
    q = ql.quantize_act_mx(X)
    want = ql.quantize_act_mx(base)
    assert torch.equal(q[0][:64], want[0]) and torch.equal(q[1][:64], want[1])
    assert periodic(torch, q[0]) and periodic(torch, q[1])
    back = ql.dequantize(ql.FMT_MXFP4, *q, dtype=torch.bfloat16)
    assert torch.equal(back[:64], ql.dequantize(ql.FMT_MXFP4, *want, dtype=torch.bfloat16))
    assert periodic(torch, back)
    del back, q
    freqs, _ = ql.rotary_frequencies(64)
    pos = torch.arange(64, device="cuda").repeat(n)
    ql.rotary(X, 512, freqs, positions=pos)
    assert torch.equal(X[:64], ql.rotary(base.clone(), 512, freqs, positions=pos[:64]))
    assert periodic(torch, X)
    del X

    N, K = 32776, 256
    rng = np.random.default_rng(2)
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32) * 0.05)
    w = dev(torch, codes), dev(torch, scales)
    x32 = rng.standard_normal((64, K)).astype(np.float32)
    xb, xv = bf16(torch, x32)
    Y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    out = lambda P, e: (P, e + R.BF16 * (np.abs(P) + e))
    for x, values in ((xb, xv), (dev(torch, x32), x32.astype(np.float64))):
        ql.forward_ep(ql.FMT_MXFP4, many(x), *w, N, Y=Y)
        check(Y[:64], *out(*R.product(values, Wv)), "product")
        assert periodic(torch, Y)
    q = ql.quantize_act_mx(xb)
    ql.forward_mx(many(q[0]), many(q[1]), *w, N, Y=Y)
    check(Y[:64], *out(*R.product(host(ql.dequantize(ql.FMT_MXFP4, *q)), Wv)), "4-bit product")
    assert periodic(torch, Y)
    X = many(xb)
    ql.gated_forward(ql.FMT_MXFP4, X, w, w, H=Y)
    check(Y[:64], *out(*R.gated(xv, Wv, Wv, 0, 0, "silu", False)[:2]), "gated")
    assert periodic(torch, Y)

    # backward, with the forward's output as dH
    b = ql.gated_backward(ql.FMT_MXFP4, X, w, w, Y, weight_grads=True, bias_grads=True)
    H, _, (G, U, eG, eU) = R.gated(xv, Wv, Wv, 0, 0, "silu", False)
    dG, dU, bG, bU = R.gated_grads(host(Y[:64]), G, U, eG, eU, "silu")
    check(b.gate[:64], dG, bG, "dG")
    check(b.up[:64], dU, bU, "dU")
    assert periodic(torch, b.gate) and periodic(torch, b.up) and periodic(torch, b.X)
    d = host(b.gate[:64]), host(b.up[:64])
    dX, S = (d[0] + d[1]) @ Wv, (np.abs(d[0]) + np.abs(d[1])) @ np.abs(Wv)
    e = S * (2 * N * R.STEP)
    check(b.X[:64], dX, e + R.BF16 * (np.abs(dX) + e), "dX")
    for got, v in ((b.W_gate, d[0]), (b.W_up, d[1])):
        dW = n * v.T @ xv
        e = M * R.STEP * n * (np.abs(v).T @ np.abs(xv))
        check(got, dW, e + R.BF16 * (np.abs(dW) + e), "dW")
    for got, v in ((b.b_gate, d[0]), (b.b_up, d[1])):
        check(got, n * v.sum(axis=0), M * R.STEP * n * np.abs(v).sum(axis=0), "db")


def test_more_rows_than_few_row_tiles(gpu):
    """More outputs than a launch of the few-row kernel could hold: the tiles take
    them."""
    torch, ql = gpu
    n, N, K = 9376, 16392, 256
    M = 64 * n
    assert (M // 16) * (N // 32) >= 1 << 24
    rng = np.random.default_rng(4)
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32) * 0.05)
    w = dev(torch, codes), dev(torch, scales)
    xb, xv = bf16(torch, rng.standard_normal((64, K)))
    X = xb.repeat(n, 1)
    Y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    q = ql.quantize_act_mx(X)
    P, e = R.product(xv, Wv)
    Pq, eq = R.product(host(ql.dequantize(ql.FMT_MXFP4, q[0][:64], q[1][:64])), Wv)
    H, eh, _ = R.gated(xv, Wv, Wv, 0, 0, "silu", False)
    for call, want, bound in (
            (lambda: ql.forward_ep(ql.FMT_MXFP4, X, *w, N, Y=Y), P, e),
            (lambda: ql.forward_mx(*q, *w, N, Y=Y), Pq, eq),
            (lambda: ql.gated_forward(ql.FMT_MXFP4, X, w, w, H=Y), H, eh)):
        Y.fill_(7)
        call()
        check(Y[:64], want, bound + R.BF16 * (np.abs(want) + bound), "first rows")
        assert periodic(torch, Y)


def test_large_weights_past_32_bits(gpu):
    """Few rows against weights of more than 2^32 bytes of codes."""
    torch, ql = gpu
    rng = np.random.default_rng(3)
    n, K = 16400, 8192
    N = 64 * n
    x32 = rng.standard_normal((3, K)).astype(np.float32)
    xb, xv = bf16(torch, x32)
    for fmt in ("mxfp4", "int8"):
        codes, scales, Wv = R.weight(fmt, rng.standard_normal((64, K)).astype(np.float32) * 0.01)
        w = tuple(dev(torch, t).repeat(n, 1) for t in (codes, scales))
        assert w[0].numel() > 1 << 32
        f = fmts(ql)[fmt]
        if fmt == "mxfp4":
            for x, values in ((xb, xv), (dev(torch, x32), x32.astype(np.float64))):
                Y = ql.forward(f, x, *w, N)
                check(Y[:, :64], *R.product(values, Wv), "product")
                assert periodic(torch, Y.t())
            q = ql.quantize_act_mx(xb)
            Y = ql.forward_mx(*q, *w, N)
            check(Y[:, :64], *R.product(host(ql.dequantize(f, *q)), Wv), "4-bit product")
            assert periodic(torch, Y.t())
        H = torch.empty((3, N), device="cuda")
        ql.gated_forward(f, xb, w, w, H=H)
        want, e, (G, U, eG, eU) = R.gated(xv, Wv, Wv, 0, 0, "silu", fmt != "mxfp4")
        check(H[:, :64], want, e, "gated")
        assert periodic(torch, H.t())
        b = ql.gated_backward(f, xb, w, w, H, dtype=torch.float32)
        dG, dU, bG, bU = R.gated_grads(host(H[:, :64]), G, U, eG, eU, "silu")
        check(b.gate[:, :64], dG, bG, "dG")
        check(b.up[:, :64], dU, bU, "dU")
        assert periodic(torch, b.gate.t()) and periodic(torch, b.up.t())
        dg, du = host(b.gate[:, :64]), host(b.up[:, :64])
        S = n * (np.abs(dg) + np.abs(du)) @ np.abs(Wv)
        check(b.X, n * (dg + du) @ Wv,
              S * (2 * N * R.STEP * (1 if fmt == "mxfp4" else 2) +
                   (R.PLANES if fmt != "mxfp4" else 0)), "dX")


# ---- together ---------------------------------------------------------------------

def block(torch, ql, seed=0, M=(2, 75), d=256, ffn=352, fmt=None):
    """The state of a small block: QKV, rotary, attention, out, gated feed-forward
    and its second half, MXFP4 weights."""
    fmt = ql.FMT_MXFP4 if fmt is None else fmt
    B, T = M
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n = lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda") * std
    w = {k: ql.quantize(fmt, n(N, K, std=K ** -0.5))
         for k, (N, K) in {"qkv": (3 * d, d), "out": (d, d), "gate": (ffn, d), "up": (ffn, d),
                           "down": (d, ffn)}.items()}
    freqs, m = ql.rotary_frequencies(32, scaling="ntk", factor=2.0)
    h = n(B * T, d)
    return dict(fmt=fmt, B=B, T=T, d=d, w=w, freqs=freqs, m=m, h=h, x=h.to(torch.bfloat16))


def run_block(torch, ql, s):
    d, w, H = s["d"], s["w"], s["d"] // 64
    qkv = ql.forward_ep(s["fmt"], s["x"], *w["qkv"], 3 * d, ydtype=torch.bfloat16)
    ql.rotary(qkv[:, :2 * d], 2 * H, s["freqs"], T=s["T"], mscale=s["m"])
    o = ql.attention(qkv[:, :d], qkv[:, d:2 * d], qkv[:, 2 * d:], s["B"], s["T"], H,
                     odtype=torch.bfloat16)
    copy = torch.empty((s["B"] * s["T"], d), dtype=torch.bfloat16, device="cuda")
    h = ql.forward_ep(s["fmt"], o, *w["out"], d, residual=s["h"], ycopy=copy)
    f = ql.gated_forward(s["fmt"], copy, w["gate"], w["up"])
    y = ql.forward_ep(s["fmt"], f, *w["down"], d, residual=h)
    g = ql.gated_backward(s["fmt"], copy, w["gate"], w["up"], f, weight_grads=True,
                          bias_grads=True)
    return [qkv, o, h, copy, f, y, *g]


def test_block_together(gpu):
    """A block of these operators against the same block in 64 bits, from each
    stage's own inputs (as the library rounded them)."""
    torch, ql = gpu
    s = block(torch, ql)
    qkv, o, h, copy, f, y = (host(t) for t in run_block(torch, ql, s)[:6])
    d, B, T, H = s["d"], s["B"], s["T"], s["d"] // 64
    W = {k: host(ql.dequantize(s["fmt"], *w)) for k, w in s["w"].items()}
    P, e = R.product(host(s["x"]), W["qkv"])
    raw = host(ql.forward_ep(s["fmt"], s["x"], *s["w"]["qkv"], 3 * d, ydtype=torch.bfloat16))
    check(raw, P, e + R.BF16 * (np.abs(P) + e), "qkv")
    pos = np.tile(np.arange(T), B)
    t, e = R.rotary(raw[:, :2 * d], 2 * H, 64, s["freqs"].cpu().numpy(), pos, False, s["m"], False)
    check(qkv[:, :2 * d], t, e + R.BF16 * (np.abs(t) + e), "rotary")
    np.testing.assert_array_equal(qkv[:, 2 * d:], raw[:, 2 * d:])
    q, k, v = (qkv[:, i * d:(i + 1) * d].reshape(B, T, H, 64).transpose(0, 2, 1, 3)
               for i in range(3))
    sc = q @ k.transpose(0, 1, 3, 2) / 8
    p = np.exp(sc - sc.max(axis=-1, keepdims=True))
    p /= p.sum(axis=-1, keepdims=True)
    a = (p @ v).transpose(0, 2, 1, 3).reshape(B * T, d)
    spread = (p @ np.abs(v)).transpose(0, 2, 1, 3).reshape(B * T, d)
    check(o, a, 2.5 * R.BF16 * spread, "attention")
    P, e = R.product(o, W["out"])
    check(h, P + host(s["h"]), e + 4 * R.F32 * (np.abs(P) + np.abs(h)), "out")
    want, e, _ = R.gated(copy, W["gate"], W["up"], 0, 0, "silu", False)
    check(f, want, e + R.BF16 * (np.abs(want) + e), "gated")
    P, e = R.product(f, W["down"])
    check(y, P + h, e + 4 * R.F32 * (np.abs(P) + np.abs(h)), "down")


def test_repeatable_on_streams(gpu):
    """The same bits on every call, on the current stream and on another."""
    torch, ql = gpu
    s = block(torch, ql, seed=3)
    first = run_block(torch, ql, s)
    again = run_block(torch, ql, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run_block(torch, ql, s)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(first, again, other):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_captured(gpu):
    """Captured into a graph and replayed, with the program's own calls and new
    inputs between the replays."""
    torch, ql = gpu
    s = block(torch, ql, seed=4, M=(1, 200))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run_block(torch, ql, s)  # the stream's workspace gets its size
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = run_block(torch, ql, s)
    for i in range(4):
        s["h"].copy_(torch.randn_like(s["h"]))
        s["x"].copy_(s["h"])
        want = run_block(torch, ql, s)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), i
        torch.ones(1000, device="cuda").sum().item()


def test_captured_without_workspace(gpu):
    """A backward pass captured on a stream that the library has not seen takes its
    workspace into the graph."""
    torch, ql = gpu
    rng, Xb, _, pair, _, _, _ = gated_case(torch, "int8", 40, 1024, 256, 6, False)
    dH = dev(torch, rng.standard_normal((40, 1024)).astype(np.float32))
    want = ql.gated_backward(ql.FMT_INT8, Xb, *pair, dH, weight_grads=True)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = ql.gated_backward(ql.FMT_INT8, Xb, *pair, dH, weight_grads=True)
    for _ in range(3):
        got.X.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got[:5], want[:5]):
            assert torch.equal(a, b)


def test_two_graphs_on_one_stream(gpu):
    """Two graphs captured on a stream share its workspace; replayed one after the
    other, with a larger call on the stream between, each gives its own results."""
    torch, ql = gpu
    cases = []
    for fmt, M, seed in (("q4", 40, 1), ("mxfp4", 130, 2)):
        rng, Xb, _, pair, _, _, _ = gated_case(torch, fmt, M, 1024, 384, seed, False)
        dH = dev(torch, rng.standard_normal((M, 1024)).astype(np.float32))
        cases.append((fmts(ql)[fmt], Xb, *pair, dH))
    call = lambda c: ql.gated_backward(*c, weight_grads=True)
    want = [call(c) for c in cases]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for c in cases:
            call(c)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in cases:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            outs.append(call(c))
    _, Xb, _, pair, _, _, _ = gated_case(torch, "int8", 700, 2048, 1024, 3, False)
    big = (ql.FMT_INT8, Xb, *pair, torch.randn((700, 2048), device="cuda"))
    big_want = call(big)
    for i in range(3):
        for k in (0, 1):
            for t in outs[k][:5]:
                t.zero_()
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                graphs[k].replay()
                got = call(big)
            torch.cuda.synchronize()
            for a, b in zip((*outs[k][:5], *got[:5]), (*want[k][:5], *big_want[:5])):
                assert torch.equal(a, b), (i, k)


def test_calls_at_once(gpu):
    """Threads with a stream each, calling at once: the same bits as alone."""
    import threading
    torch, ql = gpu
    cases = [block(torch, ql, seed=9, fmt=f, M=(1, 100 + 60 * i))
             for i, f in enumerate((ql.FMT_MXFP4, ql.FMT_Q4, ql.FMT_INT8))]
    want = [run_block(torch, ql, c) for c in cases]
    torch.cuda.synchronize()
    fails = []

    def work(k):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = run_block(torch, ql, cases[k])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[k])):
                    fails.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fails


@pytest.mark.parametrize("M,N,K", [(3, 264, 96), (40, 264, 1056), (300, 2056, 1056),
                                   (600, 4104, 288), (1100, 4104, 1056), (1100, 4104, 512)])
def test_infinities_stay_in_their_rows(gpu, M, N, K):
    """An infinity, a NaN and the largest bf16 in some rows leave every other row as it
    was; a bf16 infinity times a weight is an infinity of the product's sign, or a NaN
    for a weight of zero."""
    torch, ql = gpu
    rng = np.random.default_rng(M)
    codes, scales, Wv = R.weight("mxfp4", rng.standard_normal((N, K)).astype(np.float32) * 0.05)
    w = dev(torch, codes), dev(torch, scales)
    q4 = tuple(dev(torch, t) for t in
               R.weight("q4", rng.standard_normal((N, K)).astype(np.float32) * 0.05)[:2])
    Xb, _ = bf16(torch, rng.standard_normal((M, K)))
    bad = Xb.clone()
    rows = [0, M // 2, M - 1]
    bad[rows[0], K - 1] = float("inf")
    bad[rows[1], 5] = float("nan")
    bad[rows[2], 0] = torch.finfo(torch.bfloat16).max
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[rows] = False
    dH = torch.randn((M, N), device="cuda")
    for f in (lambda X: ql.forward(ql.FMT_MXFP4, X, *w, N),
              lambda X: ql.forward(ql.FMT_MXFP4, X.float(), *w, N),
              lambda X: ql.forward_mx(*ql.quantize_act_mx(X), *w, N),
              lambda X: ql.gated_forward(ql.FMT_MXFP4, X, w, w),
              lambda X: ql.gated_forward(ql.FMT_Q4, X, q4, q4),
              lambda X: ql.gated_backward(ql.FMT_MXFP4, X, w, w, dH).X,
              lambda X: ql.gated_backward(ql.FMT_Q4, X, q4, q4, dH).X):
        assert torch.equal(f(Xb)[rest], f(bad)[rest])
    Y = host(ql.forward(ql.FMT_MXFP4, bad, *w, N))
    with np.errstate(invalid="ignore"):
        want = np.inf * Wv[:, K - 1]
    np.testing.assert_array_equal(Y[rows[0]], want)
    assert np.isnan(Y[rows[1]]).all()
