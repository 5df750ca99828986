"""Drafted rows through ods_run_draft: attention over the paged cache and the tree masks, RoPE and KV append, against
the definitions in 64 bits, element by element, and against the decode operators where a tree is one token."""
import sys
from dataclasses import replace

import numpy as np
import pytest
import torch

import draft_ref as D
import workloads as W

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402

PAGE = 16


def say(*a):
    print("[case] tree", *a, file=sys.stderr, flush=True)


class Case:
    """A one-layer block, its pool and drafted rows; q, k, v already in qkv and the drafted keys in the pool."""

    def __init__(self, ctx, rows, n_q=4, n_kv=2, hd=64, window=0, ring=0, seed=0, max_rows=None, pad=0, chain=False,
                 extra_pages=0, std=1.0):
        self.ctx, self.n = np.asarray(ctx, np.int32), np.asarray(rows)
        self.n_q, self.n_kv, self.hd, self.window, self.ring = n_q, n_kv, hd, window, ring
        rng = self.rng = np.random.default_rng(seed)
        B = len(self.ctx)
        self.max_rows = max(1, int(self.n.max())) if max_rows is None else max_rows
        self.off = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        R_ = self.R = int(self.off[-1]) + pad
        depth, self.sets = [], []
        for n in self.n:
            d, a = D.forest(int(n), rng, 1 if chain else 4)
            depth += d
            self.sets += a
        self.depth = np.array(depth + [0] * pad, np.int32)
        self.sets += [[] for _ in range(pad)]
        cols = ring or max(1, int(max(-(-(max(int(c), 0) + int(n)) // PAGE) for c, n in zip(self.ctx, self.n)))) + extra_pages
        P = self.P = B * cols + 3
        self.table = rng.permutation(P)[:B * cols].reshape(B, cols).astype(np.int32)
        self.pool = torch.from_numpy(rng.standard_normal((P, 2, n_kv, PAGE * hd)).astype(np.float32) * std).to(torch.bfloat16)
        self.qkv = torch.from_numpy(rng.standard_normal((R_, (n_q + 2 * n_kv) * hd)).astype(np.float32)).to(torch.bfloat16)
        self.cfg = W.LayerCfg(hidden=256, n_q=n_q, n_kv=n_kv, head_dim=hd, ffn=512, window=window)

    def device(self, rope=None):
        self.dpool = self.pool.cuda()
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.block = R.DeviceBlock([self.cfg], [{}], [self.dpool], self.P)
        tab = t(self.table)
        self.batch = R.DeviceBatch(t(self.ctx), tab, ring_table=tab if self.ring else None)
        self.draft = R.DeviceDraft(t(self.off), t(self.depth), t(D.mask_words(self.sets, self.max_rows)),
                                   max_rows=self.max_rows, rope=rope)
        self.state = R.DeviceState(self.block, self.batch, fill=float("nan"), draft=self.draft)
        self.state.view("qkv", *self.qkv.shape).copy_(self.qkv)
        self.state.view("o", self.R, self.n_q * self.hd).fill_(-3.0)
        return self

    def o(self):
        return self.state.view("o", self.R, self.n_q * self.hd)

    def attend(self):
        R.run_draft(self.block, 4, 5, self.batch, self.draft, self.state)
        torch.cuda.synchronize()
        return self.o().clone()

    def expect(self, pool=None, qkv=None):
        q = (self.qkv if qkv is None else qkv)[:, :self.n_q * self.hd].double().cpu().numpy().reshape(self.R, self.n_q, self.hd)
        p = (self.pool if pool is None else pool).double().cpu().numpy()
        return D.tree_attention(q, p, self.table, self.ctx, self.off, np.clip(self.depth, 0, self.max_rows - 1), self.sets,
                                self.n_kv, self.window, self.ring, self.max_rows)

    def check(self, got, **kw):
        o, mag, touched = self.expect(**kw)
        g = got.double().cpu().numpy().reshape(o.shape)
        assert (g[~touched] == -3.0).all(), "padding rows were written"
        bound = D.tree_bound(o, mag)
        ok = (np.abs(g - o) <= bound) | (np.isnan(o) & np.isnan(g)) | (g == o)
        ok |= ~touched[:, None, None]
        bad = np.argwhere(~ok)
        assert len(bad) == 0, (f"{len(bad)} values off, first (row, head, dim) {bad[0].tolist()}: got {g[tuple(bad[0])]}, "
                               f"want {o[tuple(bad[0])]} +- {bound[tuple(bad[0])]}")


HEADS = [(4, 2, 64), (8, 1, 64), (16, 1, 128), (8, 2, 128), (3, 3, 128), (6, 2, 64)]


@pytest.mark.parametrize("n_q,n_kv,hd", HEADS)
@pytest.mark.parametrize("n", [1, 2, 5, 16, 33, 64])
def test_trees_of_every_width(n_q, n_kv, hd, n):
    say("width", n_q, n_kv, hd, n)
    ctx = [0, 1, 15, 16, 17, 31, 32, 33, 100, 511]
    c = Case(ctx, [n] * len(ctx), n_q, n_kv, hd, seed=n + hd).device()
    c.check(c.attend())


@pytest.mark.parametrize("max_rows", [65, 127, 128, 129, 200, 256])
def test_masks_of_several_words(max_rows):
    say("words", max_rows)
    c = Case([3, 40, 700], [max_rows, 66, 1], 4, 2, 64, seed=max_rows, max_rows=max_rows).device()
    c.check(c.attend())


@pytest.mark.parametrize("group,hd", [(1, 64), (2, 128), (4, 128), (7, 64), (8, 128), (16, 64), (16, 128)])
def test_ragged_batches(group, hd):
    """From no row to 70 rows a sequence, contexts from nothing to many pages, a sequence that is left alone."""
    say("ragged", group, hd)
    ctx = [0, 5, 16, -1, 47, 300, 1000, 64, 129, 2, 4000]
    rows = [3, 0, 70, 2, 1, 17, 31, 32, 33, 8, 9]
    c = Case(ctx, rows, 2 * group, 2, hd, seed=group, pad=5).device()
    c.check(c.attend())


@pytest.mark.parametrize("window", [1, 5, 16, 33, 100, 1000])
@pytest.mark.parametrize("hd", [64, 128])
def test_sliding_windows(window, hd):
    say("window", window, hd)
    c = Case([0, 3, 15, 40, 99, 100, 101, 333], [20, 9, 33, 1, 40, 7, 16, 24], 4, 2, hd, window=window, seed=window).device()
    c.check(c.attend())


@pytest.mark.parametrize("window,extra", [(20, 0), (64, 2), (100, 0)])
def test_window_rings(window, extra):
    """Slots wrap around the ring; what the ring holds of older tokens is overwritten with NaN."""
    say("ring", window)
    max_rows = 24
    ring = -(-(window + max_rows) // PAGE) + 1 + extra
    ctx = [0, 10, 50, 100, 777, 5000]
    c = Case(ctx, [24, 3, 24, 11, 1, 20], 4, 2, 64, window=window, ring=ring, seed=window, max_rows=max_rows)
    for b, x in enumerate(ctx):
        live = {(t // PAGE) % ring for t in range(max(0, x - window + 1), x + int(c.n[b]))}
        for p in range(ring):
            if p not in live:
                c.pool[c.table[b, p]] = float("nan")
    c.device()
    c.check(c.attend())


def test_masks_that_leave_rows_empty():
    """No drafted bit and no cached token: zeros. The rows' own bit is not implied."""
    say("empty")
    c = Case([0, 0, 30], [6, 40, 6], seed=4)
    for r in (0, 2, 7, 11, 45, 47):
        c.sets[r] = []
    c.sets[46] = [5, 0]                      # any set of drafted tokens, later ones too
    c.device()
    got = c.attend()
    assert (got[[0, 2, 7, 11]] == 0).all()
    c.check(got)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [7, 40])
def test_masked_slots_do_not_reach_a_row(bad, hd, rows):
    """Keys and values of a drafted token that is not an ancestor, of slots past the last token, of tokens before a
    window and of foreign pages hold infinities or NaN; rows that do see such a token get what the formula gives."""
    say("masked", bad, hd, rows)
    for window in (0, 30):
        c = Case([20, 16, 100, 0], [rows] * 4, 4, 2, hd, seed=9, window=window)
        pool = c.pool.view(c.P, 2, c.n_kv, PAGE * hd)
        seen_pages = set()
        for b, x in enumerate(c.ctx):
            for lp in range(c.table.shape[1]):
                page = int(c.table[b, lp])
                seen_pages.add(page)
                for s in range(PAGE):
                    t = lp * PAGE + s
                    if t >= x + rows or (window and t <= x - window) or t == x + 3:   # drafted token 3: seen by some rows
                        pool[page, 0, :, s * hd:(s + 1) * hd] = bad if t != x + 3 else 1.0
                        pool[page, 1, :, s::PAGE] = bad
        for page in set(range(c.P)) - seen_pages:
            pool[page] = bad
        c.device()
        c.check(c.attend())


def test_row_offsets_and_tables_the_device_should_not_have():
    """Rows past max_rows, offsets past the buffers and page ids outside the pool: in bounds, other sequences exact."""
    say("limits")
    c = Case([40, 33, 20, 50], [5, 12, 5, 4], 4, 2, 64, seed=2, max_rows=6, pad=4)
    full = c.n.copy()
    for r in range(5, 17):                  # sequence 1 has 12 rows and 6 may run
        c.sets[r] = [i for i in c.sets[r] if i < 6]
    c.depth[5:17] = np.minimum(c.depth[5:17], 5)
    c.device()
    c.table[3, 1] = c.P + 7                 # outside the pool: its tokens are skipped
    c.table[0, 0] = -1
    c.batch.page_table.copy_(torch.from_numpy(c.table))
    got = c.attend()
    c.n = np.minimum(full, 6)
    o, mag, _ = c.expect()
    g = got.double().cpu().numpy().reshape(o.shape)
    for b in range(4):
        r0 = int(c.off[b])
        rows = np.arange(r0, r0 + min(6, int(full[b])))
        if b == 1:
            assert (g[r0 + 6:r0 + 12] == -3.0).all()
            continue
        assert (np.abs(g[rows] - o[rows]) <= D.tree_bound(o[rows], mag[rows])).all(), b
    # offsets past the buffer's rows: those rows do not exist
    c.batch.page_table.copy_(torch.from_numpy(np.where((c.table < 0) | (c.table >= c.P), 0, c.table).astype(np.int32)))
    c.draft.row_off.copy_(torch.tensor([0, 5, 17, 22, 1 << 30], dtype=torch.int32))
    c.attend()
    c.draft.row_off.copy_(torch.tensor([-5, 5, 3, 1 << 30, -(1 << 31)], dtype=torch.int32))
    c.attend()


def test_tokens_past_the_page_table():
    """Drafted slots past max_pages * 16 are neither written nor attended."""
    say("past the table")
    c = Case([28, 40], [10, 3], 4, 2, 64, seed=8)
    c.table = c.table[:, :2].copy()         # 32 tokens: rows 4.. of sequence 0 have no slot; sequence 1 has a longer context
    c.device()
    got = c.attend()
    o, mag, _ = c.expect()
    g = got.double().cpu().numpy().reshape(o.shape)
    assert (np.abs(g[:10] - o[:10]) <= D.tree_bound(o[:10], mag[:10])).all()
    before = c.dpool.clone()
    R.run_draft(c.block, 3, 4, c.batch, c.draft, c.state)
    torch.cuda.synchronize()
    changed = (c.dpool != before).reshape(c.P, -1).any(dim=1).nonzero().flatten().tolist()
    assert changed == [int(c.table[0, 1])]


@pytest.mark.parametrize("std", [6.0, 30.0])
def test_sharp_scores(std):
    """Scores of tens to hundreds: the running maximum moves by many orders of magnitude."""
    say("sharp", std)
    c = Case([0, 50, 400, 3000], [9, 16, 30, 4], 8, 2, 128, seed=6, std=std).device()
    o, mag, _ = c.expect()
    g = c.attend().double().cpu().numpy().reshape(o.shape)
    # a score of size s is off by 128 * 2^-24 * sum |q k| scale <= 2^-17 * 8 * std: that much of a probability more
    more = 2.0 ** -17 * 8 * std * 2 * mag
    assert (np.abs(g - o) <= D.tree_bound(o, mag) + more).all()


def rope_of(kind, hd):
    if kind == "own":
        return None, D.freqs(hd, 1e4), hd, False, 1.0
    if kind == "part":
        return R.Rope(hd, rotary_dim=hd // 2, interleaved=True, scaling="index", factor=8.0, orig_ctx=64, amplitude=1.25), \
            D.freqs(hd // 2, 1e4, "index", 8.0, 64, 32, 1), hd // 2, True, 1.25
    return R.Rope(hd, rotary_dim=26, theta=5e5), D.freqs(26, 5e5), 26, False, 1.0


@pytest.mark.parametrize("kind", ["own", "part", "odd"])
@pytest.mark.parametrize("n_q,n_kv,hd", [(4, 2, 64), (8, 1, 128), (5, 5, 64)])
@pytest.mark.parametrize("cut", [False, True])
def test_rope_and_append(kind, n_q, n_kv, hd, cut):
    say("append", kind, n_q, n_kv, hd, cut)
    r, f, rdim, inter, amp = rope_of(kind, hd)
    c = Case([0, 5, 16, -1, 47, 300, 31], [3, 20, 40, 2, 1, 17, 16], n_q, n_kv, hd, seed=3, pad=3).device(None if r is None else [r])
    x = c.qkv.double().numpy().reshape(c.R, n_q + 2 * n_kv, hd)
    pos = np.zeros(c.R)
    live = np.zeros(c.R, bool)
    for b in range(len(c.ctx)):
        rows = slice(c.off[b], c.off[b + 1])
        pos[rows], live[rows] = c.ctx[b] + c.depth[rows], c.ctx[b] >= 0
    y = x.copy()
    y[:, :n_q + n_kv] = D.rotate(x[:, :n_q + n_kv], pos, f, rdim, inter, amp)
    bound = np.zeros_like(x)
    bound[:, :n_q + n_kv] = D.rotate_bound(x[:, :n_q + n_kv], y[:, :n_q + n_kv], rdim, inter, amp)
    y[~live], bound[~live] = x[~live], 0
    for a, e in (((2, 3), (3, 4)) if cut else ((2, 4),)):
        R.run_draft(c.block, a, e, c.batch, c.draft, c.state)
    torch.cuda.synchronize()
    got = c.state.view("qkv", c.R, n_q + 2 * n_kv, hd)
    assert (np.abs(got.double().cpu().numpy() - y) <= bound).all()
    # the pool: each drafted token's k and v bit for bit where they belong, every other slot as it was
    want = c.pool.clone()
    wv = want.view(c.P, 2, n_kv, PAGE * hd)
    g = got.cpu()
    for b in range(len(c.ctx)):
        for j in range(int(c.n[b])):
            if c.ctx[b] < 0:
                continue
            t = int(c.ctx[b]) + j
            page, s = int(c.table[b, t // PAGE]), t % PAGE
            wv[page, 0, :, s * hd:(s + 1) * hd] = g[c.off[b] + j, n_q:n_q + n_kv]
            wv[page, 1, :, s::PAGE] = g[c.off[b] + j, n_q + n_kv:]
    np.testing.assert_array_equal(D.bits(c.dpool), D.bits(want))


@pytest.mark.parametrize("hd,n_q,n_kv,window", [(64, 4, 2, 0), (128, 8, 2, 0), (128, 32, 8, 50)])
def test_one_row_is_the_decode_step(hd, n_q, n_kv, window):
    """A tree of one token at ctx is the decode operators at ctx + 1: RoPE and append bit for bit, attention within
    both sides' rounding."""
    say("decode", hd, n_q, n_kv, window)
    ctx = [0, 1, 15, 16, 100, 700]
    c = Case(ctx, [1] * len(ctx), n_q, n_kv, hd, window=window, seed=5).device()
    R.run_draft(c.block, 2, 5, c.batch, c.draft, c.state)
    pool2 = c.pool.cuda()
    block = R.DeviceBlock([c.cfg], [{}], [pool2], c.P)
    batch = R.DeviceBatch(torch.from_numpy(c.ctx + 1).cuda(), c.batch.page_table)
    st = R.DeviceState(block, batch, fill=float("nan"))
    st.view("qkv", *c.qkv.shape).copy_(c.qkv)
    R.run_partition(block, 2, 5, batch, st)
    torch.cuda.synchronize()
    assert torch.equal(c.state.view("qkv", *c.qkv.shape), st.view("qkv", *c.qkv.shape))
    assert torch.equal(c.dpool, pool2)
    qkv = st.view("qkv", *c.qkv.shape)
    c.check(c.o(), pool=pool2, qkv=qkv)
    o, mag, _ = c.expect(pool=pool2, qkv=qkv)
    d = (c.o().double() - st.view("o", *c.o().shape).double()).abs().cpu().numpy().reshape(o.shape)
    assert (d <= 2 * D.tree_bound(o, mag)).all()


def test_many_sequences():
    """More (sequence, head) pairs than waves, most of them short."""
    say("many")
    rng = np.random.default_rng(0)
    c = Case(rng.integers(0, 60, 1500), rng.integers(0, 4, 1500), 4, 2, 64, seed=1, max_rows=4).device()
    c.check(c.attend())


def test_long_context_in_a_large_pool():
    """A pool past 2^31 values and a context of 40000 tokens: offsets need 64 bits."""
    say("long")
    c = Case([40000, 17], [10, 4], 8, 2, 128, seed=3)
    o = c.expect()
    big = 270000                                            # 270000 pages * 8192 values = 2.2e9
    dpool = torch.zeros(big, 2, 2, PAGE * 128, dtype=torch.bfloat16, device="cuda")
    ids = np.sort(np.random.default_rng(1).permutation(big)[:c.P]).astype(np.int32)
    dpool[torch.from_numpy(ids.astype(np.int64)).cuda()] = c.pool.cuda()
    table = ids[c.table]
    c.device()
    c.block = R.DeviceBlock([c.cfg], [{}], [dpool], big)
    c.batch = R.DeviceBatch(c.batch.ctx_lens, torch.from_numpy(table).cuda())
    g = c.attend().double().cpu().numpy().reshape(o[0].shape)
    assert (np.abs(g - o[0]) <= D.tree_bound(o[0], o[1])).all()


@pytest.mark.parametrize("n,group,hd", [(16, 4, 128), (40, 2, 64), (3, 1, 128)])
def test_graph_replays_with_new_metadata(n, group, hd):
    """The captured range reads ctx_lens, row_off, depth and mask at launch; two graphs over one workspace replay in
    turn with eager work between, each replay equal to its eager run bit for bit."""
    say("graph", n, group, hd)
    c = Case([100, 30, 512, 0], [n, n - 1, n, n // 2 + 1], 2 * group, 2, hd, seed=7, max_rows=n).device()
    small = R.DeviceDraft(c.draft.row_off, c.draft.depth, c.draft.mask, max_rows=n)
    graphs = [R.DraftGraph(c.block, 4, 5, c.batch, c.draft, c.state), R.DraftGraph(c.block, 4, 5, c.batch, small, c.state)]
    side = torch.randn(1 << 20, device="cuda")
    for rep in range(4):
        c.ctx = np.array([100 - rep, 30, 512 - 7 * rep, 0], np.int32)
        c.batch.ctx_lens.copy_(torch.from_numpy(c.ctx))
        want = c.attend()
        c.check(want)
        for g in graphs:
            c.o().fill_(-3.0)
            side.mul_(1.0001).add_(rep)
            g.launch()
            torch.cuda.synchronize()
            assert torch.equal(c.o(), want), rep
    for g in graphs:
        g.close()


def test_streams_with_workspaces_of_their_own():
    """Two calls in flight at once on two streams, each with its own state."""
    say("streams")
    cases = [Case([900, 33, 2000], [12, 7, 16], 8, 2, 128, seed=s).device() for s in (1, 2)]
    want = [c.attend() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.o().fill_(-3.0)
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                R.run_draft(c.block, 4, 5, c.batch, c.draft, c.state)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c.o(), w)


def test_layers_of_different_shapes_share_a_call():
    """A whole block for drafted rows equals its ranges cut anywhere, and a sliding-window layer its own window."""
    say("block")
    cfg = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)
    cfgs = [replace(cfg, window=40), cfg, replace(cfg, ffn=0, n_experts=8, top_k=2, moe_ffn=128)]
    from workloads import gen
    c = Case([5, 60, 0, 200], [9, 16, 4, 1], 4, 2, 64, seed=1)
    weights = [{k: v.cuda() for k, v in gen.layer_weights(x, 1, l, "cpu", 1 / 16).items()} for l, x in enumerate(cfgs)]
    x = gen.activations(c.R, 256, 1, "cpu").cuda()
    outs = []
    for cuts in ((0, 34), (0, 2, 4, 5, 10, 12, 15, 22, 23, 24, 25, 34)):
        c.device()
        pools = [c.pool.cuda() for _ in cfgs]
        block = R.DeviceBlock(cfgs, weights, pools, c.P)
        state = R.DeviceState(block, c.batch, fill=float("nan"), draft=c.draft)
        state.view("resid", c.R, 256).copy_(x)
        for a, b in zip(cuts, cuts[1:]):
            R.run_draft(block, a, b, c.batch, c.draft, state)
        torch.cuda.synchronize()
        outs.append((state.view("resid", c.R, 256).clone(), pools))
    assert torch.isfinite(outs[0][0]).all()
    assert torch.equal(outs[0][0], outs[1][0])
    for p, q in zip(outs[0][1], outs[1][1]):
        assert torch.equal(p, q)


@pytest.mark.parametrize("batch,rows,n_kv", [(2049, 3, 1), (4096, 2, 2)])
def test_batches_of_several_launches(batch, rows, n_kv):
    """More sequences than one launch takes, some left alone, the last launch with few of them."""
    say("several launches", batch)
    rng = np.random.default_rng(batch)
    ctx = rng.integers(-1, 40, batch)
    c = Case(ctx, rng.integers(0, rows + 1, batch), 2 * n_kv, n_kv, 64, seed=1, max_rows=rows, pad=1).device()
    c.check(c.attend())


@pytest.mark.parametrize("rows", [7, 16, 30])
def test_short_contexts_in_a_wide_table(rows):
    """The launch is laid out for the table's length: most workgroups find nothing to do."""
    say("wide table", rows)
    rng = np.random.default_rng(rows)
    c = Case(rng.integers(0, 100, 32), rng.integers(1, rows + 1, 32), 16, 8, 64, seed=2, max_rows=rows, extra_pages=270).device()
    c.check(c.attend())


@pytest.mark.parametrize("n_q,hd,rows", [(2, 64, 4), (2, 128, 24), (8, 128, 40)])
def test_tables_that_end_with_the_context(n_q, hd, rows):
    """The context fills the table to a tile's end or a page past it; no drafted token has a slot."""
    say("full table", rows)
    c = Case([64, 48, 128, 16, 33], [rows, 1, rows, 3, rows], n_q, 1, hd, seed=5, max_rows=rows)
    cols = 4
    c.ctx = np.array([64, 48, 64, 16, 33], np.int32)
    c.table = np.ascontiguousarray(c.table[:, :cols])
    c.device()
    c.check(c.attend())


@pytest.mark.parametrize("batch,n_q,n_kv,hd,rows", [(160, 8, 2, 64, 8), (200, 16, 4, 64, 5), (90, 12, 3, 128, 30), (40, 16, 16, 64, 3),
                                                    (130, 6, 6, 128, 20)])
@pytest.mark.parametrize("longest", [0, 6000])
def test_more_tasks_than_workgroups(batch, n_q, n_kv, hd, rows, longest):
    """Two to four whole tasks for each workgroup, or, with one long sequence among them, tasks in several."""
    say("dealt", batch, n_kv, longest)
    rng = np.random.default_rng(batch + n_kv)
    ctx, n = rng.integers(-40, 500, batch), rng.integers(0, rows + 1, batch)
    if longest:
        ctx[batch // 3], n[batch // 3] = longest, rows
    c = Case(np.maximum(ctx, -1), n, n_q, n_kv, hd, seed=7, max_rows=rows, pad=2).device()
    c.check(c.attend())


def test_sequences_of_one_length():
    """Equal tasks, one to a workgroup and two, and a window that cuts unequal contexts to equal tasks."""
    say("equal")
    for batch, n_kv, window in ((20, 2, 0), (150, 2, 0), (64, 8, 0), (60, 4, 100)):
        ctx = np.full(batch, 300) if not window else 300 + 7 * np.arange(batch)
        c = Case(ctx, np.full(batch, 6), 2 * n_kv, n_kv, 64, window=window, seed=batch, max_rows=12).device()
        c.check(c.attend())


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [3, 7, 14, 30, 50])
def test_every_width_past_the_caches(hd, rows):
    """A table of 70000 tokens: more than the caches hold, so K and V are not read through them."""
    say("past the caches", hd, rows)
    rng = np.random.default_rng(rows)
    c = Case(rng.integers(0, 700, 8), rng.integers(1, rows + 1, 8), 8, 2, hd, seed=rows, max_rows=rows)
    c.table = np.pad(c.table, ((0, 0), (0, 4400)))
    c.device()
    c.check(c.attend())


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("batch,rows", [(5, 17), (60, 32), (1100, 32)])
def test_windows_of_wide_trees(hd, batch, rows):
    """65 to 128 query vectors per KV head in a sliding-window layer; the largest batch reads more than the caches hold."""
    say("wide windows", hd, batch, rows)
    rng = np.random.default_rng(batch)
    n = rng.integers(0, rows + 1, batch) if batch < 100 else rng.integers(0, 3, batch)
    n[0] = rows
    c = Case(rng.integers(-1, 300, batch), n, 8, 2, hd, window=100, seed=3, max_rows=rows, pad=1).device()
    c.check(c.attend())


@pytest.mark.parametrize("hd,n_q,n_kv,rows", [(64, 4, 2, 6), (128, 8, 2, 40), (128, 8, 1, 33)])
@pytest.mark.parametrize("window,ring", [(0, 0), (60, 0), (60, 9)])
def test_small_calls_in_one_launch(hd, n_q, n_kv, rows, window, ring):
    """No task can be cut: sequences that are left alone get their zeros from the same launch."""
    say("one launch", hd, rows, window, ring)
    c = Case([300, -1, 0, 40, -7, 500, -1], [rows, 3, 2, rows, rows, 1, 0], n_q, n_kv, hd, window=window, ring=ring, seed=4,
             max_rows=rows, pad=2).device()
    c.check(c.attend())
