"""Which kernels, tiles and parts the operators of include/qlinear_block.h take, on the
CPU: tests/block_probe.hip asks the library's own functions, which assume the 256
compute units of the target part where there is no GPU."""
import os
import shutil
import subprocess

import pytest

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
