"""Drafted rows over buffers that several calls share: captured graphs of different widths whose trees change, a state sized
once for the widest trees, row offsets that the device should not have, tensors that are not on the device."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402
from test_gpu_tree import Case  # noqa: E402


def say(*a):
    print("[case] reuse", *a, file=sys.stderr, flush=True)


def retree(c, rng, ctx):
    """New contexts, row counts and trees for a case that has room for max_rows rows of every sequence."""
    c.ctx = np.asarray(ctx, np.int32)
    c.n = rng.integers(0, c.max_rows + 1, len(c.ctx))
    c.off = np.concatenate([[0], np.cumsum(c.n)]).astype(np.int32)
    depth, c.sets = [], []
    for n in c.n:
        d, a = D.forest(int(n), rng, 4)
        depth += d
        c.sets += a
    pad = c.R - int(c.off[-1])
    c.depth = np.array(depth + [0] * pad, np.int32)
    c.sets += [[] for _ in range(pad)]
    c.batch.ctx_lens.copy_(torch.from_numpy(c.ctx))
    c.draft.row_off.copy_(torch.from_numpy(c.off))
    c.draft.depth.copy_(torch.from_numpy(c.depth))
    c.draft.mask.copy_(torch.from_numpy(np.ascontiguousarray(D.mask_words(c.sets, c.max_rows))))


def full(B, ctx, max_rows, n_q, n_kv, hd, seed, window=0):
    return Case(np.resize(ctx, B), [max_rows] * B, n_q, n_kv, hd, seed=seed, max_rows=max_rows, window=window).device()


@pytest.mark.parametrize("n_q,n_kv,hd,widths,window", [(8, 2, 128, (3, 16), 0), (4, 2, 64, (8, 40), 0), (8, 2, 128, (30, 70), 0),
                                                       (4, 4, 64, (1, 256), 0), (8, 2, 128, (5, 32), 60)])
def test_graphs_of_two_widths_replay_with_other_trees(n_q, n_kv, hd, widths, window):
    """Two captured ranges of different batches and query tiles over one workspace, replayed in turn: before each replay its
    contexts, row counts, depths and masks change, and eager work lies between. Every replay equals its eager run."""
    say("graphs", n_q, n_kv, hd, widths, window)
    rng = np.random.default_rng(hd + widths[1])
    cases = [full(B, [100, 30, 700, 0, 333], m, n_q, n_kv, hd, 3 + m, window) for B, m in zip((9, 4), widths)]
    ws = torch.empty(max(c.state.ws_bytes for c in cases), dtype=torch.uint8, device="cuda")
    for c in cases:
        c.state.ws = ws
        c.state.c.ws, c.state.c.ws_bytes = ws.data_ptr(), ws.numel()
    graphs = [R.DraftGraph(c.block, 4, 5, c.batch, c.draft, c.state) for c in cases]
    side = torch.randn(1 << 18, device="cuda")
    for rep in range(4):
        wants = []
        for c in cases:
            ctx = np.resize([100 - rep, 30, 700 - 90 * rep, rep, 333], len(c.ctx))
            if rep == 2:
                ctx[1] = -1
            retree(c, rng, ctx)
            c.o().fill_(-3.0)
            wants.append(c.attend())
            c.check(wants[-1])
        for c in cases:
            c.o().fill_(-3.0)
        for _ in range(2):
            for c, g in zip(cases, graphs):
                side.mul_(1.0001).add_(rep)
                ws.fill_(255)  # whatever the workspace holds
                g.launch()
        torch.cuda.synchronize()
        for c, want in zip(cases, wants):
            assert torch.equal(c.o(), want), rep
    for g in graphs:
        g.close()


@pytest.mark.parametrize("hd,n_q,n_kv", [(64, 4, 2), (128, 8, 2)])
def test_one_state_for_every_width(hd, n_q, n_kv):
    """Live buffers and workspace sized for the widest trees serve narrower ones over the same batch."""
    say("one state", hd)
    B = 32
    wide = full(B, [100, 30, 512, 0], 64, n_q, n_kv, hd, 1)
    for max_rows in (64, 33, 16, 9, 8, 4, 1):
        c = Case(np.resize([100, 30, 512, 0], B), [max_rows] * B, n_q, n_kv, hd, seed=max_rows, max_rows=max_rows,
                 extra_pages=200)
        c.device()
        wide_state = R.DeviceState(c.block, c.batch, fill=float("nan"), draft=R.DeviceDraft(
            wide.draft.row_off, wide.draft.depth, wide.draft.mask, max_rows=64))
        assert wide_state.ws_bytes >= c.state.ws_bytes and wide_state.rows >= c.draft.rows
        wide_state.view("qkv", *c.qkv.shape).copy_(c.qkv)
        wide_state.view("o", c.R, n_q * hd).fill_(-3.0)
        c.state = wide_state
        c.check(c.attend())


@pytest.mark.parametrize("off,rows", [([0, 5, 17, 22, 1 << 30], [*range(0, 11), *range(17, 28)]),
                                      ([-5, 5, 3, 1 << 30, -(1 << 31)], [*range(3, 9)]),
                                      ([30, 31, 32, 33, 34], []), ([7, 7, 7, 7, 7], []),
                                      ([29, 1 << 30, 1 << 30, -1, 4], [29])])
def test_row_offsets_the_device_should_not_have(off, rows):
    """Only rows that the offsets name, that lie in the buffers and of which a sequence has at most max_rows are touched:
    every other row of o and qkv, and every slot of the pool but those rows', stays as it was, bit for bit."""
    say("offsets", off)
    c = Case([40, 33, 20, 50], [5, 12, 5, 4], 4, 2, 64, seed=2, max_rows=6, pad=4)
    c.depth = np.minimum(c.depth, 5)
    c.device()
    assert c.R == 30
    c.draft.row_off.copy_(torch.tensor(off, dtype=torch.int32))
    other = np.setdiff1d(np.arange(c.R), rows)
    o, qkv, pool = c.attend().cpu(), c.state.view("qkv", *c.qkv.shape), c.dpool
    assert (o[other] == -3.0).all() and not (o[rows] == -3.0).all(dim=1).any()
    assert torch.isfinite(o).all()
    assert torch.equal(qkv.cpu(), c.qkv) and torch.equal(pool.cpu(), c.pool)
    R.run_draft(c.block, 2, 4, c.batch, c.draft, c.state)
    torch.cuda.synchronize()
    assert torch.equal(qkv.cpu()[other], c.qkv[other])
    slots = torch.zeros(c.P, 16, dtype=torch.bool)  # where the sequences' drafted tokens go
    for b in range(4):
        for j in range(6):
            t = int(c.ctx[b]) + j
            if t // 16 < c.table.shape[1]:
                slots[int(c.table[b, t // 16]), t % 16] = True
    changed = (pool.cpu().view(torch.int16) != c.pool.view(torch.int16)).view(c.P, 2, c.n_kv, -1)
    keys, values = changed[:, 0].view(c.P, c.n_kv, 16, 64), changed[:, 1].view(c.P, c.n_kv, 64, 16)
    assert not (keys.any(dim=3).any(dim=1) & ~slots).any() and not (values.any(dim=2).any(dim=1) & ~slots).any()
    assert bool(changed.any()) == bool(rows)


def test_tensors_that_are_not_on_the_device():
    """Refused before anything is enqueued, whichever of the call's tensors it is."""
    say("devices")
    c = Case([40, 33], [5, 3], 4, 2, 64, seed=2).device()
    cpu = lambda d: R.DeviceDraft(d.row_off.cpu(), d.depth, d.mask, d.c.max_rows)  # noqa: E731
    block = R.DeviceBlock([c.cfg], [{}], [c.pool], c.P)
    state = R.DeviceState(c.block, c.batch, device="cpu", draft=c.draft)
    batch = R.DeviceBatch(c.batch.ctx_lens, c.batch.page_table.cpu())
    for args in ((block, c.batch, c.draft, c.state), (c.block, batch, c.draft, c.state),
                 (c.block, c.batch, cpu(c.draft), c.state), (c.block, c.batch, c.draft, state)):
        with pytest.raises(ValueError, match="the host"):
            R.run_draft(args[0], 2, 5, *args[1:])
        with pytest.raises(ValueError, match="the host"):
            R.DraftGraph(args[0], 2, 5, *args[1:])
    with pytest.raises(ValueError, match="the host"):
        R.kv_copy_pages(block, torch.zeros(1, 2, dtype=torch.int32, device="cuda"))
    path, n = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="the host"):
        R.kv_accept(block, c.batch, c.draft, path, n)
    with pytest.raises(ValueError, match="the host"):
        R.kv_accept(c.block, batch, c.draft, path, n)
    c.check(c.attend())


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), 1e30])
def test_padding_rows_do_not_reach_others(fill):
    """A padded batch through dense, windowed and MoE layers: whatever the rows behind the last sequence hold, the others'
    results and the cache are the same, bit for bit."""
    say("padding", fill)
    from dataclasses import replace
    import workloads as W
    from workloads import gen
    cfg = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)
    cfgs = [cfg, replace(cfg, window=40, ffn=0, n_experts=8, top_k=2, moe_ffn=128),
            replace(cfg, ffn=0, n_experts=80, top_k=6, moe_ffn=64)]
    weights = [{k: v.cuda() for k, v in gen.layer_weights(x, 1, l, "cpu", 1 / 16).items()} for l, x in enumerate(cfgs)]
    c = Case([5, 60, 0, 200], [9, 16, 4, 1], 4, 2, 64, seed=1, pad=11).device()
    real = c.R - 11
    x = gen.activations(c.R, 256, 1, "cpu").cuda()
    outs = []
    for value in (0.0, fill):
        pools = [c.pool.cuda() for _ in cfgs]
        block = R.DeviceBlock(cfgs, weights, pools, c.P)
        state = R.DeviceState(block, c.batch, fill=value, draft=c.draft)
        state.view("resid", c.R, 256).copy_(x)[real:] = value
        R.run_draft(block, 0, block.num_ops(), c.batch, c.draft, state)
        torch.cuda.synchronize()
        outs.append((state.view("resid", c.R, 256)[:real].clone(), pools))
    assert torch.isfinite(outs[0][0]).all()
    assert torch.equal(outs[0][0], outs[1][0])
    for p, q in zip(outs[0][1], outs[1][1]):
        assert torch.equal(p.view(torch.int16), q.view(torch.int16))
