"""Groups that the page bookkeeping finds, on the host: none where nothing is shared that attention could read once."""
import numpy as np
import pytest
import torch

pytest.importorskip("paper_2609_14237_amd.binding")
from paper_2609_14237_amd import runtime as R  # noqa: E402


@pytest.mark.parametrize("rows", [0, 1, 5])
def test_no_groups_where_nothing_is_shared(rows):
    k = R.KvPages(pool_pages=100, rows=rows, max_pages=10)
    for b in range(rows):
        k.resize(b, 20 + 30 * b)
    off, tokens = k.shared()
    assert off.dtype == tokens.dtype == np.int32 and off.tolist() == [0] and tokens.tolist() == []
    s = R.SharedPrefix(torch.from_numpy(off), torch.from_numpy(tokens))
    assert s.c.n_groups == 0


@pytest.mark.parametrize("shared,groups", [(15, 0), (16, 0), (31, 0), (32, 1), (47, 1)])
def test_a_shared_tile_makes_a_group(shared, groups):
    """Attention reads whole tiles of 32 tokens once, of whole pages."""
    k = R.KvPages(pool_pages=100, rows=3, max_pages=10)
    k.resize(0, shared)
    k.fork(0, 1)
    for b, n in ((0, 100), (1, 90), (2, 64)):
        k.resize(b, n)
    off, tokens = k.shared()
    assert len(off) == len(tokens) + 1
    assert [int(t) for t in tokens if t >= 32] == [32] * groups and (len(tokens) > 0) == (groups > 0)
