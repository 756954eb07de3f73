"""A batch of no trees whose picks are given is nothing to do: no launch, no error (no GPU needed)."""
import pytest

from paper_2511_17560_amd import api

X = 0x1000          # never dereferenced on the host


@pytest.mark.parametrize("rows", [0, 1, 40, 2 ** 31 - 1])
def test_no_trees(rows):
    L = api.lib()
    call = lambda picked=X: L.a3_tree_accept(api.A3_F32, None, 0, 0, picked, X, X, 0, X, X, rows, 16, 8, X, X, X, X, X, None, 0, None)
    assert call() == api.A3_OK
    if rows:
        assert call(picked=None) == api.A3_ERR_INVALID_ARG
