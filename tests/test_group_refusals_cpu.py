"""Grouped calls of several formats on the CPU: what one layer cannot take is
refused before the layers of another format are enqueued.  (Without a GPU an
enqueued layer fails with QL_ERR_HIP, and no later one is looked at.)"""
import pytest

from paper_2607_08526_amd import qlinear as ql

OK, INVALID, SHAPE, ALIGN, RANGE, UNSUPPORTED, HIP = range(7)
A = 0x10000  # a fake, never dereferenced device address


def layer(fmt, M=4, N=64, K=1024, xdt=ql.DT_BF16):
    return ql._Linear(fmt, A, xdt, M, K, N, A, A, A)


def status(*layers):
    arr = (ql._Linear * len(layers))(*layers)
    return ql.load().qlinear_block_forward(arr, len(layers), None)


HUGE = (1 << 31) - 1


@pytest.mark.parametrize("first", [ql.FMT_Q4, ql.FMT_INT8, ql.FMT_F16])
def test_more_outputs_than_a_launch_holds(first):
    assert status(layer(ql.FMT_MXFP4, M=HUGE, N=HUGE)) == UNSUPPORTED
    assert status(layer(first), layer(ql.FMT_MXFP4, M=HUGE, N=HUGE)) == UNSUPPORTED
    assert status(layer(ql.FMT_MXFP4, M=HUGE, N=HUGE), layer(first)) == UNSUPPORTED
    assert status(layer(ql.FMT_MXFP4), layer(ql.FMT_MXFP4, M=HUGE, N=HUGE, xdt=ql.DT_F32)) == \
        UNSUPPORTED


def test_a_forced_kernel_that_a_format_cannot_take():
    with ql.forced_path(ql.PATH_MID):
        assert status(layer(ql.FMT_INT8, K=96)) == UNSUPPORTED
        assert status(layer(ql.FMT_Q4), layer(ql.FMT_INT8, K=96)) == UNSUPPORTED
        assert status(layer(ql.FMT_INT8, K=96), layer(ql.FMT_Q4)) == UNSUPPORTED
