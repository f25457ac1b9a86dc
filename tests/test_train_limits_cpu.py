"""The masked attention's limits on its number of workgroups, on the CPU: calls past them are
refused before anything is launched."""
import pytest

from test_train_cpu import OK, UNSUPPORTED, attend, attend_back, lib  # noqa: F401


@pytest.mark.parametrize("B, Tk", [(1 << 24, 1), (1 << 25, 1), (1 << 23, 129), (1 << 20, 1921)])
def test_backward_without_queries(lib, B, Tk):  # noqa: F811
    """Without queries only kept keys make workgroups: one for each 128 of a sequence."""
    how = dict(B=B, H=1, Hk=1, Tq=0, Tk=Tk, q_rows=0, k_rows=B * Tk, k=1 << 50, v=1 << 52)
    far = dict(dk=1 << 54, dv=1 << 56, lddk=64, lddv=64, ldo=64, lddo=64, lddq=64)
    assert attend_back(lib, **how, **far) == UNSUPPORTED
    assert attend(lib, **how, ldo=64) == OK  # nothing to do


def test_forward_of_many_sequences(lib):  # noqa: F811
    how = dict(H=1, Hk=1, Tk=1, Tq=1, q=1 << 50, k=1 << 52, v=1 << 54)
    B = 1 << 24
    assert attend(lib, **how, B=B, q_rows=B, k_rows=B) == UNSUPPORTED
    assert attend(lib, **{**how, "Tq": 33}, B=B // 2, q_rows=33 * B // 2,
                  k_rows=B // 2) == UNSUPPORTED
