"""Scratch memory of the orthogonalised updates, on the CPU."""
import pytest

from paper_2501_08582_amd import _lib

AT = 1 << 40


@pytest.mark.parametrize("side", [1, 16, 17, 48, 64, 65, 96, 97, 128])
@pytest.mark.parametrize("long", [128, 1000, 70000])
def test_a_matrix_s_scratch_is_a_multiple_of_256_bytes(side, long):
    """So that each of a call's matrices, and their table behind them, starts at one of the workspace's."""
    p = _lib.Update(0.9, 1e-7, 3.4445, -4.775, 2.0315, 5, 1, _lib.DTYPE_BF16, _lib.DTYPE_BF16, 0)
    items = (_lib.UpdateItem * 2)(*((side, long, AT, AT, AT, AT, 0.1, 0.0),) * 2)
    one = _lib.orthogonal_workspace_bytes(p, items, 1)
    assert one % 256 == 0 and _lib.orthogonal_workspace_bytes(p, items, 2) == 2 * one
