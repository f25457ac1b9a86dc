"""How the masked attention cuts its work, on the CPU: tests/train_probe.hip asks the
library's own functions, which assume the 256 compute units of the target part where
there is no GPU."""
import math
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_train_attention as A

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
BUILD = os.path.join(ROOT, "paper_2607_08526_amd", "_build")


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
    for cmd in ([hipcc, *flags, "-c", os.path.join(HERE, "train_probe.hip"), "-o", obj],
                [hipcc, "--offload-arch=gfx950", "-o", exe, obj, *objs]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]

    def run(kind, cases):
        lines = [f"{kind} {c['B']} {c['T']} {c.get('kT', c['T'])} {c['H']} {c.get('Hk', c['H'])} "
                 f"{c['dh']} {int(c['causal'])} {c.get('more', '')}" for c in cases]
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True,
                           timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return [tuple(map(int, l.split()[1:])) for l in r.stdout.strip().splitlines()]
    return run


def all_of(shapes):
    return [dict(s, dh=dh, causal=c) for s in shapes for dh in (64, 128) for c in (False, True)]


def test_forms_that_the_gpu_tests_run(probe):
    """Every number of groups, unsplit and in parts, at both head sizes, and parts of both
    passes backward: what a call can reach, the GPU tests run."""
    cases = all_of(A.FORWARD + A.LENGTHS) + [dict(A.LARGE, dh=64, causal=False)]
    seen = {(c["dh"], g, s > 1) for c, (g, s, _, _) in zip(cases, probe("fwd", cases))}
    assert seen == {(dh, g, s) for dh in (64, 128) for g in (1, 2, 4) for s in (False, True)}
    cases = all_of([s for s in A.FORWARD if s["B"] * s["T"] * s["H"] < 9000] + A.LENGTHS)
    plans = list(zip(cases, probe("bwd", cases)))
    for dh in (64, 128):
        assert {q > 1 for c, (q, _, _, _) in plans if c["dh"] == dh} == {False, True}
        assert {k > 1 for c, (_, k, _, _) in plans if c["dh"] == dh} == {False, True}


def test_workspace_of_split_work(probe):
    """The bounds that the header states, over random calls of every size."""
    rng = random.Random(4)
    log = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    cases = []
    while len(cases) < 4000:
        Hk = log(1, 64)
        c = dict(B=log(1, 512), T=log(1, 100000), kT=log(1, 2000000), H=Hk * log(1, 16), Hk=Hk,
                 dh=rng.choice([64, 128]), causal=rng.random() < 0.5)
        rows = -(-c["T"] * (c["H"] // Hk) // 32)
        if c["B"] * c["H"] * c["T"] < 1 << 31 and c["B"] * Hk * c["kT"] < 1 << 31 and \
                c["B"] * Hk * rows < 1 << 24:
            cases.append(c)
    for c, (groups, splits, wgs, size) in zip(cases, probe("fwd", cases)):
        assert size <= 80 << 20, c
        assert (size == 0) == (splits == 1) and (splits == 1 or wgs <= 1024), c
        assert groups in (1, 2, 4) and splits <= max(1, -(-c["kT"] // 64)), c
    for c, (qparts, kparts, wgs, size) in zip(cases, probe("bwd", cases)):
        assert size <= 160 << 20, c  # (no rows here: nothing for the sums)
        assert qparts <= 16 and kparts <= 16, c


def test_plans_of_measured_calls(probe):
    """Calls that were measured in every form (a change of the estimates that flips one is
    to be measured)."""
    case = lambda B, T, kT, H, Hk, dh, causal=False: dict(B=B, T=T, kT=kT, H=H, Hk=Hk, dh=dh,
                                                          causal=causal)
    got = probe("fwd", [case(1, 4096, 4096, 32, 32, 64), case(2, 645, 77, 24, 24, 64),
                        case(3, 592, 592, 8, 8, 64, True), case(2, 107, 107, 24, 24, 64)])
    assert [g[:2] for g in got] == [(1, 1), (1, 1), (2, 1), (2, 1)]
    got = probe("bwd", [case(1, 4096, 4096, 32, 32, 64), case(1, 2048, 2048, 32, 8, 128, True),
                        case(3, 778, 778, 8, 8, 64, True)])
    assert [g[:2] for g in got] == [(1, 1), (1, 4), (1, 1)]


def test_order_of_work(probe):
    """Every part of every block of every unit is some workgroup's, once, in any order."""
    rng = random.Random(5)
    cases = []
    while len(cases) < 300:
        B, Hk = rng.choice([1, 1, 2, 3, 8, 25]), rng.choice([1, 2, 5, 8, 16, 32])
        parts, blocks = rng.choice([1, 1, 2, 3, 8]), rng.randint(1, 70)
        if B * Hk * parts * blocks <= 6000:
            cases.append(dict(B=B, T=1, H=Hk, Hk=Hk, dh=64, causal=rng.random() < 0.7,
                              more=f"{parts} {blocks} {rng.choice([1, 2])}", size=(parts, blocks)))
    seen = set()
    for c, (fold, group, *work) in zip(cases, probe("work", cases)):
        parts, blocks = c["size"]
        units = c["B"] * c["Hk"]
        work = list(zip(work[::3], work[1::3], work[2::3]))
        assert sorted(work) == [(p, b, u) for p in range(parts) for b in range(blocks)
                                for u in range(units)], c
        assert c["causal"] or (fold, group) == (0, 1)
        seen.add((fold, group > 1, group > 1 and units // 8 % group > 0 and units // 8 > group))
        if group > 1:  # of an XCD's units that are taken together, the longest first
            for xcd in range(8):
                blks = [b for _, b, _ in work[xcd::8]][: parts * blocks * min(group, units // 8)]
                assert blks == sorted(blks), c
    assert seen >= {(0, False, False), (1, False, False), (0, True, False), (0, True, True)}
