"""Which kernels, tiles and parts the operators of include/qlinear_block.h take, on the
CPU: tests/block_probe.hip asks the library's own functions, which assume the 256
compute units of the target part where there is no GPU."""
import math
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_block as B
import test_gpu_block_variants as V

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
BUILD = os.path.join(ROOT, "paper_2607_08526_amd", "_build")
MX, Q4, INT8 = 20, 4, 8
FMTS = {"mxfp4": MX, "q4": Q4, "int8": INT8}
A16, A2 = 16, 18  # addresses of scales


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("hipcc is not available")
    objs = [os.path.join(BUILD, f) for f in sorted(os.listdir(BUILD))
            if f.endswith(".o")] if os.path.isdir(BUILD) else []
    if not objs:
        pytest.fail("library objects missing: run `python -m paper_2607_08526_amd.build`")
    out = tmp_path_factory.mktemp("probe")
    obj, exe = str(out / "probe.o"), str(out / "probe")
    flags = ["--offload-arch=gfx950", "-O1", "-std=c++17", f"-I{os.path.join(ROOT, 'include')}",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
    for cmd in ([hipcc, *flags, "-c", os.path.join(HERE, "block_probe.hip"), "-o", obj],
                [hipcc, "--offload-arch=gfx950", "-o", exe, obj, *objs]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]

    def run(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True,
                           timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return [l.split()[1:] for l in r.stdout.strip().splitlines()]
    return run


def grads(probe, calls):
    """calls: (fmt, M, N, K) or with the scales' address -> (direct, dX rows, parts,
    workgroups, dW rows, parts, workgroups)"""
    out = probe([f"grad {FMTS[c[0]]} {c[1]} {c[2]} {c[3]} {c[4] if len(c) > 4 else A16}"
                 for c in calls])
    return [tuple(map(int, t)) for t in out]


def test_backward_plans_of_measured_products(probe):
    """The plans of the large backward passes that were measured in every number of
    parts (a change of the estimate's constants that flips one is to be measured)."""
    got = grads(probe, [("mxfp4", 2048, 4096, 1536), ("mxfp4", 2048, 5504, 2048),
                        ("mxfp4", 2048, 2048, 1024), ("q4", 107, 2752, 1024),
                        ("q4", 2048, 5504, 2048)])
    assert got == [(0, 128, 5, 480, 128, 1, 384),  # dX in 2 parts 9.7 us slower, in 4 2.0
                   (0, 128, 4, 512, 128, 1, 688),  # in 2 parts 4.7 us slower
                   (0, 64, 2, 256, 64, 1, 256),    # in 4 parts of either 1.4 us faster
                   (1, 64, 20, 160, 128, 1, 176),
                   (0, 128, 4, 512, 128, 1, 688)]  # in 2 parts 18 us slower


def layers(probe, calls):
    """calls: (fmt, fp32 X, gated, epilogue, M, N, K) -> the kernel's instance and shape:
    the few-row kernel; the K-group kernel by rows staged and shape; tiles by their rows,
    wide scales and epilogue"""
    out = probe([f"rows {FMTS[f]} {int(x)} {int(g)} {M} {M} {N} {K}"
                 for f, x, g, _, M, N, K in calls])
    res = []
    for (f, x, g, e, M, N, K), t in zip(calls, out):
        if t[0] == "kgm":
            staged = "f32" if x else next(r for r in (8, 16, 32, 1 << 31) if M <= r)
            res.append((f, x, g, "kgm", staged, int(t[1])))
        elif t[0] == "tile":
            wide = K % (512 if f == "mxfp4" else 256) == 0
            res.append((f, g, "tile", int(t[1]), wide, e and not g))
        else:
            res.append((f, x, g, "any"))
    return res


def products4(probe, calls):
    """calls: (epilogue, act, M, N, K) of 4-bit activations -> as layers()"""
    out = probe([f"mx4 {int(e)} {int(a)} {M} {N} {K}" for e, a, M, N, K in calls])
    return [(int(t[1]), K % 512 == 0, e or a) if t[0] == "tile" else
            (1 if M <= 16 else 2 if M <= 32 else 4)
            for (e, a, M, N, K), t in zip(calls, out)]


def backward(probe, calls):
    """calls: (fmt, M, N, K) -> of each the instance that forms dX, and the one of dW"""
    res = []
    for (f, _, _, _), (direct, xr, xp, xw, wr, wp, ww) in zip(calls, grads(probe, calls)):
        res.append(("direct", f, xr, xp > 1) if direct else
                   ("dX", f == "mxfp4", xr, xw <= 256, xp > 1))
        res.append(("dW", wr, ww <= 256, wp > 1))
    return res


def epilogue_shapes():
    for mark in B.test_mx_epilogue.pytestmark:
        if mark.name == "parametrize" and mark.args[0] == "M,N,K":
            return mark.args[1]


class Draws:
    def __init__(self, seed):
        self.r = random.Random(seed)

    def log(self, lo, hi):
        return int(round(math.exp(self.r.uniform(math.log(lo), math.log(hi)))))

    def size(self):
        """M, N, K of models' layers, and of vocabularies at few rows"""
        K = 32 * self.log(1, 512) if self.r.random() < 0.5 else 256 * self.log(1, 64)
        if self.r.random() < 0.1:
            return self.log(1, 32), self.log(4096, 300000), K
        return self.log(1, 8192), self.log(1, 16384), K


def test_gpu_tests_run_every_layer_variant(probe):
    d = Draws(1)
    kinds = [("mxfp4", 0, 0, 0), ("mxfp4", 0, 0, 1), ("mxfp4", 1, 0, 0), ("mxfp4", 0, 1, 0),
             ("q4", 0, 1, 0), ("int8", 0, 1, 0)]
    reached = set(layers(probe, [(*d.r.choice(kinds), *d.size()) for _ in range(40000)]))
    run = [("mxfp4", x, 0, 0, *s) for s in B.SHAPES for x in (0, 1)]
    run += [("mxfp4", 0, 0, 1, *s) for s in epilogue_shapes()]
    run += [("mxfp4", int(x == "f32"), 0, 0, *s) for x, *s in V.PRODUCTS]
    run += [(f, 0, 1, 0, *s) for s in B.GATED for f in FMTS]
    run += [(f, 0, 1, 0, *s) for f, *s in V.GATED]
    assert len(reached) > 60
    assert reached - set(layers(probe, run)) == set()


def test_gpu_tests_run_every_4_bit_variant(probe):
    d = Draws(2)
    reached = set(products4(probe, [(e := d.r.randrange(2), e and d.r.randrange(2), *d.size())
                                    for _ in range(10000)]))
    run = [(0, 0, *s) for s in B.SHAPES] + [(1, a, *s) for s in epilogue_shapes() for a in (0, 1)]
    assert len(reached) == 3 + 8
    assert reached - set(products4(probe, run)) == set()


def test_gpu_tests_run_every_backward_variant(probe):
    d = Draws(3)
    calls = [(d.r.choice(list(FMTS)), *d.size()) for _ in range(20000)]
    reached = set(backward(probe, [(f, M, 8 * (N // 8) + 8, K) for f, M, N, K in calls]))
    run = [(f, *s) for s in B.GATED if s[1] % 8 == 0 for f in FMTS] + V.BACKWARD
    run += [c for c in V.GATED if c[2] % 8 == 0 and c[1] < 100]
    assert len(reached) > 30
    assert reached - set(backward(probe, run)) == set()
