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
