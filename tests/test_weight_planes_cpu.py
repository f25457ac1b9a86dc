"""The two bf16 that a q4 or int8 weight c * s enters a product as, on the CPU over
every code and every fp16 mantissa: their sum is off by at most what the header
states, both have the weight's sign, and neither is zero where the weight is not."""
import numpy as np
import pytest


def truncated(v):
    return (v.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)


def nearest(v):
    u = v.view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)
    return u.astype(np.uint32).view(np.float32)


def planes(c, s):
    """hi, lo of code c and (fp16) scale s by the kernels' steps in fp32."""
    step_up = (s.astype(np.float32).view(np.uint32) | np.uint32(1)).view(np.float32)
    v = c.astype(np.float32) * step_up
    hi = truncated(v)
    return hi, nearest(v - hi)


# normal scales, and the subnormal ones (fewer bits)
SCALES = {e: (np.arange(1024, 2048) * 2.0 ** e).astype(np.float16) for e in (-24, -14, 0, 5)}
SCALES["subnormal"] = (np.arange(1, 1024) * 2.0 ** -24).astype(np.float16)


@pytest.mark.parametrize("bits,bound", [(4, 2.0 ** -22), (8, 2.0 ** -16)])
@pytest.mark.parametrize("e", list(SCALES))
def test_every_weight(bits, bound, e):
    c = np.arange(-(1 << (bits - 1)), 1 << (bits - 1))[:, None]
    s = SCALES[e][None, :]
    hi, lo = planes(c, s)
    w = c.astype(np.float64) * s.astype(np.float64)
    off = np.abs(hi.astype(np.float64) + lo.astype(np.float64) - w)
    assert (off <= bound * np.abs(w)).all()
    assert (np.sign(hi) == np.sign(w)).all() and (np.sign(lo) == np.sign(w)).all()
    with np.errstate(invalid="ignore"):
        x = np.float32(np.inf)
        np.testing.assert_array_equal(x * lo + x * hi, (np.inf * w).astype(np.float32))


def test_scale_of_zero():
    """A zero block gives zeros whatever its codes are: the step on zero is too small
    for a bf16."""
    hi, lo = planes(np.arange(-128, 128)[:, None], np.zeros((1, 1), np.float16))
    assert not hi.any() and not lo.any()
