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
