"""The operators of include/qlinear_block.h where calls meet each other or the
ends of their ranges: threads on one stream, infinite activations, far positions."""
import ctypes
import threading

import numpy as np
import pytest

import block_ref as R
from test_gpu_block import check, dev, fmts, gated_case, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def test_threads_on_one_stream(gpu):
    """Threads that call on the same stream share its workspace: each backward pass
    (partial sums and weights in bf16 there) and large product (activations there)
    still gives what it gives alone."""
    torch, ql = gpu
    calls = []
    for fmt, M, N, K, seed in (("q4", 40, 1024, 384, 1), ("int8", 700, 1024, 256, 2),
                               ("mxfp4", 600, 2048, 512, 3)):
        rng, Xb, _, pair, _, _, _ = gated_case(torch, fmt, M, N, K, seed, False)
        dH = dev(torch, rng.standard_normal((M, N)).astype(np.float32))
        calls.append(lambda f=fmts(ql)[fmt], X=Xb, p=pair, d=dH: ql.gated_backward(
            f, X, *p, d, weight_grads=True)[:5])
    codes, scales = ql.quantize(ql.FMT_Q4, torch.randn((1024, 512), device="cuda"))
    X = torch.randn((1100, 512), device="cuda").to(torch.bfloat16)
    calls.append(lambda: [ql.forward(ql.FMT_Q4, X, codes, scales, 1024)])
    want = [c() for c in calls]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    fails = []

    def work(k):
        with torch.cuda.stream(stream):
            for _ in range(40):
                got = calls[k]()
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[k])):
                    fails.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fails


def test_outputs_of_another_stream(gpu):
    """Outputs that a call on another stream makes do not take memory that the
    current stream's queue may still use: a block freed there stays away from them,
    and they have the values of a call on the current stream."""
    torch, ql = gpu
    rng, Xb, _, pair, _, _, db = gated_case(torch, "q4", 64, 256, 128, 5, True)
    dH = dev(torch, rng.standard_normal((64, 256)).astype(np.float32))
    W = dev(torch, rng.standard_normal((256, 128)).astype(np.float32))
    mx = ql.quantize(ql.FMT_MXFP4, W)
    q = ql.quantize_act_mx(Xb)
    q8 = ql.quantize_act(Xb)
    w8 = ql.quantize(ql.FMT_INT8, W)
    calls = [lambda s: ql.gated_forward(ql.FMT_Q4, Xb, *pair, bias=db, stream=s),
             lambda s: ql.gated_backward(ql.FMT_Q4, Xb, *pair, dH, bias=db, weight_grads=True,
                                         bias_grads=True, stream=s),
             lambda s: ql.forward_mx(*q, *mx, 256, stream=s),
             lambda s: ql.quantize_act_mx(Xb, stream=s),
             lambda s: ql.dequantize(ql.FMT_MXFP4, *mx, stream=s),
             lambda s: ql.quantize(ql.FMT_MXFP4, W, stream=s),
             lambda s: ql.forward(ql.FMT_MXFP4, Xb, *mx, 256, stream=s),
             lambda s: ql.forward_ep(ql.FMT_Q4, Xb, *pair[0], 256, stream=s),
             lambda s: ql.quantize_act(Xb, stream=s),
             lambda s: ql.forward_w8a8(*q8, *w8, 256, stream=s),
             lambda s: ql.attention(Xb[:, :64], Xb[:, :64], Xb[:, 64:], 1, 64, 1, stream=s)]
    side = torch.cuda.Stream()
    for i, call in enumerate(calls):
        tensors = lambda r: [r] if isinstance(r, torch.Tensor) else list(r)
        want = [t.clone() for t in tensors(call(None))]  # its own outputs are free again
        torch.cuda.synchronize()
        gone = [torch.empty_like(t) for t in want]
        freed = {t.data_ptr() for t in gone}
        del gone
        got = tensors(call(side))
        side.synchronize()
        for a, b in zip(got, want):
            assert a.data_ptr() not in freed, i
            assert torch.equal(a, b), i


def exact_turn(freqs, positions):
    """cos and sin [position][frequency] of the exact product of both: 60 digits down
    to less than a turn."""
    import math
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi2 = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    out = np.empty((2, len(positions), len(freqs)))
    for i, p in enumerate(positions):
        for j, f in enumerate(freqs):
            turns = Decimal(int(p)) * Decimal(float(f)) / pi2
            t = float((turns - turns.to_integral_value()) * pi2)
            out[:, i, j] = math.cos(t), math.sin(t)
    return out


@pytest.mark.parametrize("rot", [64, 20])  # whole vectors, and pair by pair
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_far_positions(gpu, rot, interleaved):
    """Positions at both ends of the range: angles as exact there as near zero.  Of
    (1, 0) the turned pair is cosine and sine themselves.  Rounding the reduced angle
    (at most half a turn) to fp32 is off by 2^-26 of a turn, below 2^-23; sine and
    cosine of it by two steps of values up to 1, 2^-23."""
    torch, ql = gpu
    rng = np.random.default_rng(rot)
    far = 1 << 31
    pos = np.concatenate([[0, 1, -1, far, far - 1, -far, 1 - far, (1 << 30) + 7],
                          rng.integers(far - (1 << 20), far, 8), rng.integers(-far, far, 8)])
    freqs = rng.uniform(0.5, 1.0, rot // 2)  # (radians per position)
    freqs[-3:] = [1.0, 2.0 * np.pi, 1e-5]
    x = torch.zeros((len(pos), 64), device="cuda")
    a = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    b = a + (1 if interleaved else rot // 2)
    x[:, a] = 1.0
    c, s = exact_turn(freqs, pos)
    for adjoint in (False, True):
        y = host(ql.rotary(x, 1, dev(torch, freqs), positions=dev(torch, pos),
                           interleaved=interleaved, adjoint=adjoint, out=torch.empty_like(x)))
        check(y[:, a], c, 2.0 ** -22, "cosine")
        check(y[:, b], -s if adjoint else s, 2.0 ** -22, "sine")
    # rows that count from a start
    y = host(ql.rotary(x[:4], 1, dev(torch, freqs), start=far - 2, T=3, interleaved=interleaved,
                       out=torch.empty_like(x[:4])))
    c, s = exact_turn(freqs, [far - 2, far - 1, far, far - 2])
    check(y[:, a], c, 2.0 ** -22, "cosine")
    check(y[:, b], s, 2.0 ** -22, "sine")


# ---- the values that q4 and int8 weights have in the products ----------------------

PLANES = {"q4": 2.0 ** -22, "int8": 2.0 ** -16, "mxfp4": 0.0}  # of a weight, at most


def every_weight(torch, fmt):
    """(codes, scales, 64-bit values) [1024][256]: every code with every fp16 mantissa,
    exponents in turn (MXFP4: every code with scale bytes 97 to 160)."""
    rng = np.random.default_rng(0)
    N, K = 1024, 256
    if fmt == "mxfp4":
        c = np.tile(np.arange(16), (N, K // 16)).astype(np.uint8)
        s = (97 + np.arange(N * (K // 32)) % 64).reshape(N, K // 32).astype(np.uint8)
        return dev(torch, R.pack4(c)), dev(torch, s), R.mx_decode(c, s)
    s = np.repeat(np.arange(1024, 2048) * 2.0 ** (np.arange(N) % 12 - 18.0), K // 32)
    s = s.reshape(N, K // 32).astype(np.float16)
    lo, hi = (-8, 8) if fmt == "q4" else (-128, 128)
    c = np.tile(np.arange(lo, hi), (N, K // (hi - lo))).astype(np.int8)
    c = c[:, rng.permutation(K)]
    packed = R.pack4(c.view(np.uint8) & 15) if fmt == "q4" else c.view(np.uint8)
    return dev(torch, packed), dev(torch, s.view(np.int16)), R.int_decode(c, s)


@pytest.mark.parametrize("fmt", ["q4", "int8", "mxfp4"])
@pytest.mark.parametrize("M", [1, 8, 16, 40, 256, 700, 2048, 6144])
@pytest.mark.parametrize("narrow", [False, True])
def test_every_weight_forward(gpu, fmt, M, narrow):
    """Rows of the identity (and rows with an infinity in its place) against weights of
    every code and mantissa, U = 1: H is the weight as the kernel has it, plus zeros;
    an infinity of its sign, NaN for a zero.  narrow: K = 224, where scales of a row
    come one by one (and short reductions)."""
    torch, ql = gpu
    codes, scales, W = every_weight(torch, fmt)
    K = 224 if narrow else 256
    if narrow:
        codes = codes[:, :codes.shape[1] * 7 // 8].contiguous()
        scales = scales[:, :7].contiguous()
        W = W[:, :K]
    zero = (torch.zeros_like(codes), torch.zeros_like(scales) + (127 if fmt == "mxfp4" else 0))
    bias = (torch.zeros(1024, device="cuda"), torch.ones(1024, device="cuda"))
    rng = np.random.default_rng(M)
    k = torch.from_numpy(rng.permutation(np.arange(max(M, K)) % K)[:M]).cuda()
    want = W.T[k.cpu().numpy()]
    X = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    rows = torch.arange(M, device="cuda")
    X[rows, k] = 1.0
    # (one product, its planes and zeros: no sum rounds but the planes' own, 2^-24; the
    # bias and the product with 1 keep it)
    H = ql.gated_forward(fmts(ql)[fmt], X, (codes, scales), zero, bias=bias, act=ql.ACT_NONE,
                         hdtype=torch.float32)
    check(H, want, (PLANES[fmt] + R.F32) * np.abs(want), "weights")
    # an infinity: both projections see it, the up projection's zeros give NaN; so the
    # weights in both, and H = G U = infinity squared, or NaN
    X[rows, k] = float("inf")
    H = host(ql.gated_forward(fmts(ql)[fmt], X, (codes, scales), (codes, scales),
                              act=ql.ACT_NONE, hdtype=torch.float32))
    want = np.where(W == 0, np.nan, np.inf)
    np.testing.assert_array_equal(H, want.T[k.cpu().numpy()])


@pytest.mark.parametrize("fmt", ["q4", "int8", "mxfp4"])
@pytest.mark.parametrize("M", [8, 107, 500, 1024])
def test_every_weight_backward(gpu, fmt, M):
    """dX of rows of the identity (and of infinities), G = U = 1: twice the weight as
    the kernel has it, an infinity of its sign, NaN for a zero."""
    torch, ql = gpu
    codes, scales, W = every_weight(torch, fmt)
    N, K = W.shape
    one = torch.ones(N, device="cuda")
    n = torch.from_numpy(np.random.default_rng(M).permutation(N)[:M]).cuda()
    rows = torch.arange(M, device="cuda")
    X = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    dH = torch.zeros((M, N), device="cuda")
    pair = (codes, scales), (codes, scales)
    call = lambda: ql.gated_backward(fmts(ql)[fmt], X, *pair, dH, bias=(one, one), act=ql.ACT_NONE,
                                     dtype=torch.float32)
    want = 2 * W[n.cpu().numpy()]
    dH[rows, n] = 1.0
    check(call().X, want, (PLANES[fmt] + 2 * R.F32) * np.abs(want), "weights")
    dH[rows, n] = float("inf")
    # (0 * inf: the other weights of the reduction meet zeros, not infinities)
    with np.errstate(invalid="ignore"):
        np.testing.assert_array_equal(host(call().X), np.inf * want)


def test_stream_per_thread(gpu):
    """hipStreamPerThread is one handle for a stream of each thread: calls of several
    threads on it do not share a workspace."""
    torch, ql = gpu

    class PerThread:
        cuda_stream = 2  # hipStreamPerThread

    calls = []
    for fmt, M, N, K, seed in (("q4", 40, 1024, 384, 1), ("int8", 700, 1024, 256, 2),
                               ("mxfp4", 600, 2048, 512, 3)):
        rng, Xb, _, pair, _, _, _ = gated_case(torch, fmt, M, N, K, seed, False)
        dH = dev(torch, rng.standard_normal((M, N)).astype(np.float32))
        both = torch.empty((2, M, N), dtype=torch.bfloat16, device="cuda")
        dX = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
        g, _, _, _, keep = ql._gated(fmts(ql)[fmt], Xb, *pair, None, ql.ACT_SILU)
        d = ql._GatedGrad(dH.data_ptr(), ql.DT_F32, both[0].data_ptr(), both[1].data_ptr(),
                          dX.data_ptr(), ql.DT_BF16, None, None, 0, None, None)
        calls.append((g, d, dX, (keep, dH, both),
                      ql.gated_backward(fmts(ql)[fmt], Xb, *pair, dH).X))
    torch.cuda.synchronize()
    fails = []
    lib = ql.load()

    def work(k):
        g, d, dX, _, want = calls[k]
        torch.cuda.set_device(0)
        for _ in range(40):
            if lib.qlinear_gated_backward(ctypes.byref(g), ctypes.byref(d),
                                          ql._stream(PerThread())) != 0:
                fails.append((k, "status"))
            torch.cuda.synchronize()
            if not torch.equal(dX, want):
                fails.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fails
