"""Frequencies of rotary positions at long trained contexts, on the CPU."""
import math

import pytest
import torch

from paper_2607_08526_amd import qlinear as ql


def yarn(rot, base, factor, context):
    """Frequencies and turns within the context, pair by pair, from the definition:
    pair j turns context base^(-2 j / rot) / 2 pi times; the ramp runs from the last
    pair that turns at least 32 times to the first that turns at most once, counting
    on past the last pair where that one still turns more than once (to place
    rot - 1)."""
    turns = lambda j: context * base ** (-2 * j / rot) / (2 * math.pi)
    lo = max([j for j in range(rot) if turns(j) >= 32], default=0)
    hi = min([j for j in range(rot) if turns(j) <= 1], default=rot - 1)
    out = []
    for j in range(rot // 2):
        f = base ** (-2 * j / rot)
        w = min(max((j - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
        out.append(f * (1 - w) + f / factor * w)
    return out, [turns(j) for j in range(rot // 2)]


@pytest.mark.parametrize("rot,base", [(64, 10000.0), (128, 10000.0), (32, 500000.0), (8, 100.0)])
@pytest.mark.parametrize("context", [256, 4096, 65536, 131072, 1 << 20, 1 << 26])
@pytest.mark.parametrize("factor", [1.0, 4.0, 16.0])
def test_yarn_at_long_contexts(rot, base, context, factor):
    got, m = ql.rotary_frequencies(rot, base=base, scaling="yarn", factor=factor, context=context,
                                   device="cpu")
    want, turns = yarn(rot, base, factor, context)
    assert got.shape == (rot // 2,) and m == 0.1 * math.log(factor) + 1
    # (both in 64 bits: a few roundings of each)
    assert torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=1e-13, atol=0)
    f = ql.rotary_frequencies(rot, base=base, device="cpu")[0]
    for j, t in enumerate(turns):
        if t >= 32:
            assert got[j] == f[j]
        elif t > 1 and factor > 1:  # never divided in full
            assert got[j] > f[j] / factor * (1 + 1e-9)


def test_yarn_of_the_slowest_pair():
    """rot 64, base 10000, factor 4, trained on 131072: the ramp runs over pairs 22 to
    35, so the last pair, which turns 2.8 times, is 9 / 13 of the way to a quarter."""
    f = ql.rotary_frequencies(64, device="cpu")[0]
    y = ql.rotary_frequencies(64, scaling="yarn", factor=4.0, context=131072, device="cpu")[0]
    assert abs(y[-1] / f[-1] - (1 - 0.75 * 9 / 13)) < 1e-12
