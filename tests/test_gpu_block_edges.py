"""The operators of include/qlinear_block.h where calls meet each other or the
ends of their ranges: threads on one stream, infinite activations, far positions."""
import threading

import numpy as np
import pytest

import block_ref as R
from test_gpu_block import acts, bf16, check, dev, fmts, gated_case, host

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
