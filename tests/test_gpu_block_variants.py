"""The kernels' shapes, tiles and parts that the sizes of test_gpu_block.py do not
reach, against the same 64-bit references, with the bounds of q4 and int8 weights
of each format.  tests/test_block_plans_cpu.py holds that the two files together
run every variant that a call can reach."""
import numpy as np
import pytest

import block_ref as R
import test_gpu_block as B
from test_gpu_block import check, dev, fmts, gated_case, host
from test_gpu_block_edges import PLANES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


@pytest.fixture
def planes(monkeypatch):
    return lambda fmt: monkeypatch.setattr(R, "PLANES", PLANES[fmt])


PRODUCTS = [("bf16", 2, 8797, 864), ("bf16", 2, 17265, 800), ("bf16", 9, 9343, 800),
            ("bf16", 9, 17143, 800), ("bf16", 17, 9275, 864), ("bf16", 17, 17003, 992),
            ("bf16", 171, 3730, 512), ("f32", 1416, 1521, 512)]
GATED = [("mxfp4", 3, 8504, 2080), ("mxfp4", 11, 9352, 2080), ("mxfp4", 3, 16700, 2080),
         ("mxfp4", 11, 16700, 2080), ("mxfp4", 25, 1008, 832), ("mxfp4", 25, 16733, 1056),
         ("mxfp4", 4422, 136, 544), ("mxfp4", 1094, 1040, 1536), ("q4", 10, 10457, 1056),
         ("q4", 9, 16968, 1056), ("q4", 19, 8789, 800), ("q4", 18, 17431, 1024),
         ("q4", 640, 1595, 544), ("q4", 2, 9576, 1120), ("q4", 2, 16480, 1056),
         ("int8", 9, 12144, 1056), ("int8", 18, 8433, 800), ("int8", 2, 9757, 1056)]
# dX from the compressed weights and from their bf16 copy, dW: both tiles, one and
# several parts, a workgroup for each CU or more
BACKWARD = [("int8", 5776, 128, 608), ("mxfp4", 2709, 128, 1408), ("mxfp4", 4273, 968, 96),
            ("q4", 2974, 128, 2688), ("mxfp4", 4342, 128, 1824), ("mxfp4", 5862, 5416, 96),
            ("int8", 144, 4080, 2592), ("mxfp4", 5413, 5352, 128), ("mxfp4", 1130, 2704, 96),
            ("int8", 22, 8472, 288), ("mxfp4", 2341, 8728, 96), ("mxfp4", 773, 128, 96),
            ("q4", 3221, 5400, 96), ("mxfp4", 68, 3352, 2432)]


@pytest.mark.parametrize("x,M,N,K", PRODUCTS)
def test_product(gpu, x, M, N, K):
    B.test_mx_product(gpu, M, N, K, x)


@pytest.mark.parametrize("fmt,M,N,K", GATED)
def test_forward(gpu, planes, fmt, M, N, K):
    planes(fmt)
    B.test_gated_forward(gpu, fmt, M, N, K)


@pytest.mark.parametrize("dhdt", ["f32", "bf16"])
@pytest.mark.parametrize("fmt,M,N,K", [c for c in GATED if c[2] % 8 == 0 and c[1] < 100])
def test_backward_of_gated(gpu, planes, fmt, M, N, K, dhdt):
    planes(fmt)
    B.test_gated_backward(gpu, fmt, M, N, K, dhdt)


@pytest.mark.parametrize("i", range(len(BACKWARD)))
def test_backward(gpu, planes, i):
    fmt, M, N, K = BACKWARD[i]
    planes(fmt)
    B.test_gated_backward(gpu, fmt, M, N, K, ("f32", "bf16")[i % 2])


@pytest.mark.parametrize("fmt", ["mxfp4", "q4", "int8"])
@pytest.mark.parametrize("M,N,K", [(3, 72, 96), (40, 264, 1056), (300, 1032, 384),
                                   (1100, 2056, 288), (1100, 2056, 512)])
@pytest.mark.parametrize("which", ["gate", "up", "both", "neither"])
def test_one_bias(gpu, planes, fmt, M, N, K, which):
    """A pair with a bias on one projection alone, and no activation: forward and
    backward."""
    torch, ql = gpu
    planes(fmt)
    rng, Xb, Xv, pair, (Wg, Wu), b, db = gated_case(torch, fmt, M, N, K, M + K, True)
    has = [which in ("gate", "both"), which in ("up", "both")]
    bias = tuple(d if h else None for d, h in zip(db, has))
    b = [v if h else np.zeros(N) for v, h in zip(b, has)]
    H, e, (G, U, eG, eU) = R.gated(Xv, Wg, Wu, *b, "none", fmt != "mxfp4")
    kw = dict(bias=bias, act=ql.ACT_NONE)
    check(ql.gated_forward(fmts(ql)[fmt], Xb, *pair, hdtype=torch.float32, **kw), H, e, "H")
    dH = rng.standard_normal((M, N)).astype(np.float32)
    g = ql.gated_backward(fmts(ql)[fmt], Xb, *pair, dev(torch, dH), weight_grads=True,
                          bias_grads=True, dtype=torch.float32, **kw)
    dG, dU, bG, bU = R.gated_grads(dH.astype(np.float64), G, U, eG, eU, "none")
    check(g.gate, dG, bG, "dG")
    check(g.up, dU, bU, "dU")
    d = host(g.gate), host(g.up)
    S = np.abs(d[0]) @ np.abs(Wg) + np.abs(d[1]) @ np.abs(Wu)
    terms = 2 * N * (1 if fmt == "mxfp4" else 2)
    check(g.X, d[0] @ Wg + d[1] @ Wu, S * (terms * R.STEP + PLANES[fmt]), "dX")
    for got, v in ((g.W_gate, d[0]), (g.W_up, d[1])):
        check(got, v.T @ Xv, M * R.STEP * (np.abs(v).T @ np.abs(Xv)), "dW")
    for got, v in ((g.b_gate, d[0]), (g.b_up, d[1])):
        check(got, v.sum(axis=0), M * R.STEP * np.abs(v).sum(axis=0), "db")
