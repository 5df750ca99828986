"""Token counts of the page bookkeeping that no 32-bit argument holds."""
import numpy as np
import pytest

B = pytest.importorskip("paper_2609_14237_amd.binding")
from paper_2609_14237_amd import runtime as R  # noqa: E402


@pytest.mark.parametrize("tokens", [1 << 31, 1 << 32, (1 << 32) + 16, (1 << 32) + 33, -1, -(1 << 31) - 1, 16 - (1 << 32), 1 << 63])
def test_token_counts_that_wrap_are_refused(tokens):
    k = R.KvPages(8, 2, 4)
    k.resize(0, 40)
    before = k.table.copy(), k.tokens.copy(), k._refs.copy(), k.free
    with pytest.raises((ValueError, B.OdsError)):
        k.resize(0, tokens)
    for a, b in zip(before, (k.table, k.tokens, k._refs, k.free)):
        np.testing.assert_array_equal(a, b)
    k.resize(0, np.int64(64))
    assert k.tokens[0] == 64 and (k.table[0] >= 0).all()
