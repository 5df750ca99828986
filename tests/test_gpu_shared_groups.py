"""Groups of a shared prefix whose members are not alike: some left alone, released or shorter than what the group shares, the
first one above all."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402
from test_gpu_shared import PAGE, Shared, cuda  # noqa: E402


def say(*a):
    print("[case] groups", *a, file=sys.stderr, flush=True)


@pytest.mark.parametrize("n_q,n_kv,hd", [(8, 2, 128), (4, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("ends", ["left alone", "released", "shorter", "no rows", "all but one", "none has it"])
def test_first_members_without_the_prefix(ends, n_q, n_kv, hd):
    """What the others share is read by the table of one that has it, wherever in the group that is."""
    say(ends, n_q, n_kv, hd)
    ctx, rows = [200, 230, 192, 260, 301, 96, 120, 97], [2, 1, 2, 1, 2, 1, 2, 1]
    first = {"all but one": 4, "none has it": 5}.get(ends, 1)
    for b in range(first):
        if ends == "shorter" or ends == "none has it":
            ctx[b] = 40 + b
        elif ends == "no rows":
            rows[b] = 0
        else:
            ctx[b] = -1
    c = Shared([(5, 192), (3, 96)], ctx, rows, n_q=n_q, n_kv=n_kv, hd=hd, seed=first, max_rows=2)
    for b in range(first):
        if ends in ("released", "no rows"):
            c.table[b] = -1
        elif ends != "left alone":               # the table names pages as far as the sequence goes
            c.table[b, max(-(-(ctx[b] + rows[b]) // PAGE), 0):] = -1
    c.device()
    c.check(c.attend())
    c.device(shared=False)
    c.check(c.attend())


def test_members_that_end_between_replays():
    """A captured call: the first sequences of a group end one after the other, their tables with them."""
    say("graph")
    c = Shared([(6, 320)], [330, 350, 325, 400, 321, 500], [1, 2, 1, 2, 2, 1], n_q=8, n_kv=2, hd=128, seed=20).device()
    g = R.DraftGraph(c.block, 4, 5, c.batch, c.draft, c.state)
    for b in range(6):
        c.o().fill_(-3.0)
        g.launch()
        torch.cuda.synchronize()
        got = c.o().clone()
        c.check(got)
        c.o().fill_(-3.0)
        assert torch.equal(c.attend(), got)
        c.ctx[b] = -1
        c.table[b] = -1
        c.batch.ctx_lens.copy_(cuda(c.ctx))
        c.batch.page_table[b].fill_(-1)
    g.close()


def test_first_members_without_the_prefix_on_both_sides_of_a_launch():
    """More sequences than a launch takes: on either side of the border the group's first ones have no table."""
    say("launches")
    B = 530
    ctx, rows = 64 + np.arange(B) % 9, np.ones(B, np.int64)
    ctx[:3] = ctx[512:515] = -1
    c = Shared([(B, 64)], ctx, rows, n_q=4, n_kv=2, hd=64, seed=21)
    c.table[:3] = c.table[512:515] = -1
    c.device()
    c.check(c.attend())


def test_rows_that_descend_share_nothing():
    """Offsets of rows that do not ascend, so that the rows of one group's sequences lie among those another group's offsets
    span: every sequence that has rows of its own gets its own attention, and nothing else is written."""
    say("rows")
    ctx = [200 + 7 * b for b in range(8)]
    for off in ([0, 3, 12, 24, 6, 9, 12, 0, 0], [6, 9, 0, 24, 3, 9, 24, 12, 15], [0, 3, 6, 9, 12, 15, 18, 21, 24]):
        c = Shared([(2, 192), (2, 64), (2, 192), (2, 96)], ctx, [3] * 8, n_q=8, n_kv=2, hd=64, seed=22, pad=4)
        c.device()
        c.off = np.array(off, np.int32)
        c.draft.row_off[:9].copy_(cuda(c.off))
        c.draft.row_off[9:].fill_(int(c.off[-1]))
        guard = 1 << 16
        ws = torch.full((c.state.ws_bytes + 2 * guard,), 0x5a, dtype=torch.uint8, device="cuda")
        c.state.c.ws = ws.data_ptr() + guard
        c.check(c.attend())
        assert (ws[:guard] == 0x5a).all() and (ws[guard + c.state.ws_bytes:] == 0x5a).all()


@pytest.mark.parametrize("B,size,tokens", [(1500, 3, 64), (4096, 9, 32), (1100, 40, 96)])
def test_groups_on_both_sides_of_a_launch(B, size, tokens):
    """The sequences around every border between launches, and the last ones, against the definition."""
    say("border", B, size)
    rng = np.random.default_rng(B)
    ctx, rows = tokens + rng.integers(0, 40, B), rng.integers(0, 3, B)
    c = Shared([(size, tokens)] * (B // size), ctx, rows, n_q=4, n_kv=1, hd=64, seed=B, max_rows=2).device()
    assert len(c.tokens) <= 512
    got = c.attend().double().cpu().numpy().reshape(c.R, 4, 64)
    pool = c.pool.double().numpy()
    q = c.qkv[:, :256].double().numpy().reshape(c.R, 4, 64)
    near = {b for at in [*range(512, B, 512), B] for b in range(at - size - 1, min(at + size + 1, B))}
    for b in sorted(near):
        a, e = int(c.off[b]), int(c.off[b + 1])
        if a == e:
            continue
        o, mag, _ = D.tree_attention(q[a:e], pool, c.table[b:b + 1], c.ctx[b:b + 1], [0, e - a], c.depth[a:e], c.sets[a:e], 1)
        off = np.abs(got[a:e] - o) - D.tree_bound(o, mag)
        assert (off <= 0).all(), f"sequence {b}: off by {off.max()} more than the bound"
