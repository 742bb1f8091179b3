"""Positions of another shape than the rows and the axes of a rotation are refused by the binding.  CPU only: nothing may
reach the library."""
import pytest

from test_more_readouts_abi import D, H, MN, b, bf, calls, f32, there  # noqa: F401 (b and calls are fixtures)


def spec(rs3, axes):
    s = rs3.rope_spec(D)
    s.axes, s.rot = axes, D
    return s


def rows(rs3, pos, axes):
    x, y = there(1, MN, H * D, dtype=bf), there(1, MN, H * D, dtype=bf)
    rs3.rs3_rope_rows(x, y, pos, None, None, None, "bf16", H, 0, D, spec(rs3, axes))


def keys(rs3, pos, axes):
    x, y = there(1, MN, H * D, dtype=bf), there(1, MN, H * D, dtype=bf)
    rs3.rs3_rope_rows(None, None, None, x, y, pos, "bf16", 0, H, D, spec(rs3, axes))


def table(rs3, pos, axes):
    rs3.rs3_rope_table(pos, spec(rs3, axes), there(4 * MN, D // 2, 2, dtype=f32))


@pytest.mark.parametrize("axes,shape", [(1, (MN,)), (1, (MN, 1)), (2, (MN, 2)), (2, (1, MN, 2)), (3, (4, MN // 4, 3))])
@pytest.mark.parametrize("call", [rows, keys, table])
def test_positions_of_every_row_reach_the_library(calls, call, axes, shape):
    rs3, reached, _, _ = calls
    call(rs3, there(*shape), axes)
    assert len(reached) == 1


@pytest.mark.parametrize("axes,shape", [(2, (MN, 3)), (2, (MN, 1)), (1, (MN, 2)), (3, (MN, 2)), (2, (2 * MN,)), (2, (3 * MN,)),
                                        (3, (3, MN)), (2, (2, MN)), (2, ()), (1, ())])
@pytest.mark.parametrize("call", [rows, keys, table])
def test_positions_of_other_axes_are_refused(calls, call, axes, shape):
    rs3, reached, _, _ = calls
    with pytest.raises(ValueError, match="pos"):
        call(rs3, there(*shape), axes)
    assert not reached


def test_one_axis_may_be_left_out(calls):
    """Of rows, whose number says how many there are; a table's rows are those of a list."""
    rs3, reached, _, _ = calls
    for call in (rows, keys):
        call(rs3, there(1, MN), 1)
    assert len(reached) == 2
    with pytest.raises(ValueError, match="pos"):
        table(rs3, there(1, MN), 1)


@pytest.mark.parametrize("axes,shape", [(1, (MN + 1,)), (2, (MN - 1, 2)), (2, (MN + 1, 2)), (3, (2, MN, 3))])
@pytest.mark.parametrize("call", [rows, keys])
def test_positions_of_other_rows_are_refused(calls, call, axes, shape):
    rs3, reached, _, _ = calls
    with pytest.raises(ValueError, match="pos"):
        call(rs3, there(*shape), axes)
    assert not reached
