"""Without a GPU: a call on more rows than its state's live buffers hold is refused on the host, where alone their sizes are
known. The block has no weights, so no call here could reach a launch."""
import pytest
import torch

import workloads as W

B = pytest.importorskip("paper_2609_14237_amd.binding")
from paper_2609_14237_amd import runtime as R  # noqa: E402

CFG = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)


def z(*shape, dt=torch.int32):
    return torch.zeros(*shape, dtype=dt)


def draft_of(batch, rows, max_rows=64):
    return R.DeviceDraft(z(batch + 1), z(rows), z(rows, dt=torch.int64), max_rows=max_rows)


def setup(batch=2, rows=None):
    block = R.DeviceBlock([CFG], [{}], [None], 0)
    b = R.DeviceBatch(z(batch), z(batch, 4))
    draft = None if rows is None else draft_of(batch, rows)
    return block, b, R.DeviceState(block, b, device="cpu", draft=draft)


def test_drafted_rows_past_the_state():
    block, batch, state = setup(2, rows=8)
    assert state.rows == 8
    for ops in ((0, 10), (2, 5), (4, 5), (5, 6)):
        with pytest.raises(ValueError, match="9 rows"):
            R.run_draft(block, *ops, batch, draft_of(2, 9), state, stream=0)
        with pytest.raises(ValueError, match="9 rows"):
            R.DraftGraph(block, *ops, batch, draft_of(2, 9), state)
        for rows in (8, 3):  # these get as far as the library's own checks
            with pytest.raises(B.OdsError):
                R.run_draft(block, *ops, batch, draft_of(2, rows), state, stream=0)
    # a state that was made for a batch of single tokens
    block, batch, state = setup(4)
    assert state.rows == 4
    with pytest.raises(ValueError, match="5 rows"):
        R.run_draft(block, 2, 5, batch, draft_of(4, 5), state, stream=0)


def test_batches_past_the_state():
    block, _, state = setup(2)
    more = R.DeviceBatch(z(3), z(3, 4))
    for call in (lambda: R.run_partition(block, 0, 10, more, state, stream=0),
                 lambda: R.run_partition_scratch(block, 0, 10, more, state, stream=0),
                 lambda: R.attn_stage(block, 0, more, state, stream=0),
                 lambda: R.ffn_stage(block, 0, more, state, stream=0),
                 lambda: R.PartitionGraph(block, 0, 10, more, state)):
        with pytest.raises(ValueError, match="3 rows"):
            call()
    with pytest.raises(B.OdsError):
        R.run_partition(block, 0, 10, R.DeviceBatch(z(2), z(2, 4)), state, stream=0)


def test_contexts_for_every_sequence():
    """row_off and the page table name three sequences, ctx_lens two."""
    block, _, state = setup(3, rows=8)
    batch = R.DeviceBatch(z(2), z(3, 4))
    with pytest.raises(ValueError, match="ctx_lens"):
        R.run_draft(block, 2, 5, batch, draft_of(3, 8), state, stream=0)
    with pytest.raises(ValueError, match="ctx_lens"):
        R.kv_accept(block, batch, draft_of(3, 8), z(3, 4), z(3), stream=0)
