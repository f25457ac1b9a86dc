"""qlinear_gated_backward refuses an output at the address of any input or other
output, on the CPU (fake addresses, never dereferenced)."""
import ctypes
import itertools

import pytest

from paper_2607_08526_amd import qlinear as ql

OK, INVALID, HIP = 0, 1, 6
INPUTS = ["X", "gate_codes", "gate_scales", "up_codes", "up_scales", "gate_bias", "up_bias", "dH"]
OUTPUTS = ["dG", "dU", "dX", "dWg", "dWu", "dbg", "dbu"]


def status(M=4, **at):
    p = {n: 0x100000 * (i + 1) for i, n in enumerate(INPUTS + OUTPUTS)} | at
    g = ql._Gated(ql.FMT_MXFP4, p["X"], M, 64, 16, p["gate_codes"], p["gate_scales"], p["up_codes"],
                  p["up_scales"], p["gate_bias"], p["up_bias"], ql.ACT_SILU)
    d = ql._GatedGrad(p["dH"], ql.DT_F32, p["dG"], p["dU"], p["dX"], ql.DT_BF16, p["dWg"], p["dWu"],
                      ql.DT_F32, p["dbg"], p["dbu"])
    return ql.load().qlinear_gated_backward(ctypes.byref(g), ctypes.byref(d), None)


def address(name):
    return 0x100000 * ((INPUTS + OUTPUTS).index(name) + 1)


@pytest.mark.parametrize("out,other", list(itertools.product(OUTPUTS, INPUTS)) +
                         list(itertools.combinations(OUTPUTS, 2)))
def test_same_address(out, other):
    assert status(**{out: address(other)}) == INVALID
    # without rows only the gradients of weights and biases are written
    written = {"dWg", "dWu", "dbg", "dbu"}
    if out in written and (other in written or other in INPUTS[1:7]):
        assert status(M=0, **{out: address(other)}) == INVALID
