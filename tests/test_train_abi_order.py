"""CPU test of the C ABI of the operators around the layer: a norm of no known kind is
refused where formats are, before shapes and after dtypes."""
import pytest

from paper_2501_08582_amd import _lib
from test_train_abi import BAD, call_norm_backward, call_norm_forward, norm, ptrs


@pytest.mark.parametrize("kind", [-1, 2])
def test_kind_before_shape(kind):
    for call, n in ((call_norm_forward, 8), (call_norm_backward, 10)):
        for wrong in (dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(p=2.0)):
            assert call(norm(kind=kind, **wrong), ptrs(n)) == _lib.ERR_UNSUPPORTED, wrong
            assert call(norm(**wrong), ptrs(n)) == _lib.ERR_SHAPE, wrong
        assert call(norm(kind=kind, dtype=9), ptrs(n)) == _lib.ERR_DTYPE
    assert _lib.norm_workspace_bytes(norm(kind=kind)) == BAD
