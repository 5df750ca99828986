"""Page copies and accepted paths against the definition, bit for bit over the whole pools."""
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
CFG = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)


def say(*a):
    print("[case] pages", *a, file=sys.stderr, flush=True)


def raw_pools(cfgs, P, seed):
    """Pools of random bit patterns (NaN among them): moves keep bits."""
    g = np.random.default_rng(seed)
    return [torch.from_numpy(g.integers(-32768, 32768, (P, 2, c.n_kv, PAGE * c.head_dim)).astype(np.int16))
            .view(torch.bfloat16).cuda() for c in cfgs]


@pytest.mark.parametrize("heads", [(1, 64), (2, 64), (3, 128), (8, 128)])
@pytest.mark.parametrize("n,layers", [(0, 1), (1, 1), (5, 3), (70, 2), (333, 1), (9, 35)])
def test_copies(n, layers, heads):
    say("copy", n, layers, heads)
    P = 2 * n + 20
    cfgs = [replace(CFG, n_q=heads[0], n_kv=heads[0], head_dim=heads[1])] * layers
    pools = raw_pools(cfgs, P, n)
    rng = np.random.default_rng(n)
    ids = rng.permutation(P).astype(np.int32)
    src, dst = ids[:n], ids[n:2 * n]
    if n > 5:
        src[3] = src[2]                                       # one page copied twice
    extra = np.array([[P, 0], [-1, 0], [0, P + 9], [0, -(1 << 31)], [ids[-1], ids[-1]]], np.int32)  # skipped
    pairs = np.concatenate([np.stack([src, dst], 1), extra])
    want = [D.bits(p) for p in pools]
    for w in want:
        w[dst] = w[src]
    block = R.DeviceBlock(cfgs, [{}] * layers, pools, P)
    R.kv_copy_pages(block, torch.from_numpy(pairs).cuda())
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        np.testing.assert_array_equal(D.bits(p), w)


def test_copies_of_some_layers_and_pool_sizes():
    """Layers of different shapes and pool sizes; a pair outside the smaller pool is skipped there."""
    say("layers")
    cfgs = [CFG, replace(CFG, n_kv=4), replace(CFG, head_dim=128), CFG]
    pools = raw_pools(cfgs, 30, 3)
    pools[2] = pools[2][:20].clone()
    block = R.DeviceBlock(cfgs, [{}] * 4, pools, [30, 30, 20, 30])
    want = [D.bits(p) for p in pools]
    for l in (1, 2):
        want[l][4] = want[l][7]
        if l == 1:
            want[l][25] = want[l][3]
    R.kv_copy_pages(block, torch.tensor([[7, 4], [3, 25]], dtype=torch.int32, device="cuda"), layers=(1, 3))
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        np.testing.assert_array_equal(D.bits(p), w)


class Kept:
    def __init__(self, ctx, rows, cfgs, seed, cols=40, window_ring=0, max_rows=None, path_cols=None):
        rng = np.random.default_rng(seed)
        self.ctx, self.n, self.cfgs = np.asarray(ctx, np.int32), np.asarray(rows), cfgs
        B = len(self.ctx)
        self.off = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.max_rows = max_rows or max(1, int(self.n.max()))
        need = int(max(-(-(max(int(c), 0) + int(n)) // PAGE) for c, n in zip(ctx, rows))) or 1
        self.P = B * max(need, window_ring or 0) + 3
        self.table = rng.permutation(self.P)[:B * need].reshape(B, need).astype(np.int32)
        self.ring = window_ring
        self.ring_table = rng.permutation(self.P)[:B * window_ring].reshape(B, window_ring).astype(np.int32) if window_ring else None
        self.pools = raw_pools(cfgs, self.P, seed)
        w = path_cols or max(1, int(max(rows)))
        self.path = np.cumsum(rng.integers(1, 4, (B, w)), axis=1).astype(np.int32) - 1
        self.len = rng.integers(0, w + 1, B).astype(np.int32)

    def run(self, ctx_out=True, layers=None, alias=False):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        R_ = int(self.off[-1])
        words = (self.max_rows + 63) // 64
        self.block = R.DeviceBlock(self.cfgs, [{}] * len(self.cfgs), self.pools, self.P)
        self.batch = R.DeviceBatch(t(self.ctx), t(self.table), ring_table=None if self.ring_table is None else t(self.ring_table))
        self.draft = R.DeviceDraft(t(self.off), torch.zeros(R_, dtype=torch.int32).cuda(),
                                   torch.zeros(R_, words, dtype=torch.int64).cuda(), max_rows=self.max_rows)
        out = self.batch.ctx_lens if alias else torch.full((len(self.ctx),), -9, dtype=torch.int32, device="cuda")
        want = [D.bits(p) for p in self.pools]
        a, b = layers or (0, len(self.cfgs))
        tables = [self.ring_table if c.window and self.ring else self.table for c in self.cfgs]
        rings = [self.ring if c.window and self.ring else 0 for c in self.cfgs]
        new = D.accept(want[a:b], tables[a:b], rings[a:b], self.ctx, self.off, self.path, self.len,
                       [c.n_kv for c in self.cfgs[a:b]], [c.head_dim for c in self.cfgs[a:b]])
        R.kv_accept(self.block, self.batch, self.draft, t(self.path), t(self.len), ctx_out=out if ctx_out else None, layers=layers)
        torch.cuda.synchronize()
        for l, (p, w) in enumerate(zip(self.pools, want)):
            np.testing.assert_array_equal(D.bits(p), w, err_msg=f"layer {l}")
        if ctx_out:
            np.testing.assert_array_equal(out.cpu().numpy(), new)


@pytest.mark.parametrize("heads", [(1, 64), (2, 64), (2, 128), (8, 128)])
@pytest.mark.parametrize("rows", [1, 2, 7, 16, 33, 64, 130, 256])
def test_accepted_paths(rows, heads):
    say("accept", rows, heads)
    cfgs = [replace(CFG, n_q=heads[0], n_kv=heads[0], head_dim=heads[1])] * 2
    ctx = [0, 1, 15, 16, 17, 31, 100, -1]
    k = Kept(ctx, [rows] * len(ctx), cfgs, rows)
    k.len[:3] = k.path.shape[1], 1, 0
    k.run()


def test_accept_everything_and_nothing():
    say("accept all")
    k = Kept([5, 30, 16], [20, 20, 20], [CFG], 1)
    k.path[:] = np.arange(20)               # the whole chain: nothing moves
    k.len[:] = 20
    before = D.bits(k.pools[0])
    k.run()
    np.testing.assert_array_equal(D.bits(k.pools[0]), before)
    k.len[:] = 0, -5, -(1 << 31)
    k.run()


def test_paths_that_end_early():
    """Not ascending, repeated, negative, past the rows, lengths past the columns."""
    say("accept cut")
    k = Kept([5, 30, 16, 40, 7, 9, 9], [20] * 7, [CFG, replace(CFG, head_dim=128)], 2, path_cols=6)
    k.path[:] = [[1, 4, 4, 9, 12, 15], [2, 5, 3, 9, 12, 15], [-1, 4, 6, 9, 12, 15], [1, 19, 20, 21, 22, 23],
                 [3, 4, 6, 9, 12, 15], [1 << 30, 4, 6, 9, 12, 15], [0, 1, 2, 7, -7, 15]]
    k.len[:] = 6, 6, 6, 6, 1 << 30, 6, 6
    k.run()


def test_accept_more_than_a_wave_of_entries():
    say("accept long")
    k = Kept([3, 300], [256, 256], [CFG], 4, path_cols=200)
    k.path[:] = np.arange(200) + np.arange(200) // 4
    k.len[:] = 200
    k.path[1, 131] = 3
    k.run()


def test_accept_rings_layers_and_contexts_in_place():
    say("accept ring")
    window, rows = 40, 24
    ring = -(-(window + rows) // PAGE) + 1
    cfgs = [replace(CFG, window=window), CFG, replace(CFG, window=window, head_dim=128)]
    ctx = [0, 13, 100, 250, 95]
    for kw in (dict(), dict(alias=True), dict(ctx_out=False), dict(layers=(1, 3)), dict(layers=(0, 1), alias=True)):
        k = Kept(ctx, [rows] * 5, cfgs, 8, window_ring=ring, max_rows=rows)
        k.len[:] = 7, 24, 8, 1, 11
        k.run(**kw)


def test_accept_across_many_layers():
    say("accept 35 layers")
    k = Kept([20, 3], [9, 9], [CFG] * 35, 9)
    k.len[:] = 5, 9
    k.run()


def test_accept_rows_without_pages():
    """Slots past the table or on pages outside the pool stay where they are; the context still counts them."""
    say("accept pages")
    k = Kept([10, 40, 12], [30, 30, 30], [CFG], 10)
    k.table = np.ascontiguousarray(k.table[:, :4])
    k.table[0, 1] = -1
    k.table[2, 2] = k.P + 3
    k.len[:] = 14, 14, 14
    k.run()


@pytest.mark.parametrize("rows", [6, 40])
def test_accept_and_copy_in_a_graph(rows):
    """Captured by torch and replayed on new paths and contexts, contexts updated in place."""
    say("accept graph")
    k = Kept([20, 33, 5], [rows] * 3, [CFG, CFG], 12)
    k.run()                                  # warm: also builds the device structures
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    path, ln = t(k.path), t(k.len)
    pairs = torch.tensor([[int(k.table[0, 0]), k.P - 1]], dtype=torch.int32, device="cuda")
    used = set(k.table.flatten().tolist())
    spare = next(p for p in range(k.P) if p not in used)
    pairs[0, 1] = spare
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        R.kv_copy_pages(k.block, pairs)
        R.kv_accept(k.block, k.batch, k.draft, path, ln, ctx_out=k.batch.ctx_lens)
    rng = np.random.default_rng(3)
    for rep in range(4):
        k.ctx = rng.integers(0, 30, 3).astype(np.int32)
        k.len = rng.integers(0, rows + 1, 3).astype(np.int32)
        k.path = (np.cumsum(rng.integers(1, 4, k.path.shape), axis=1) - 1).astype(np.int32)
        k.batch.ctx_lens.copy_(t(k.ctx)); path.copy_(t(k.path)); ln.copy_(t(k.len))
        torch.cuda.synchronize()
        want = [D.bits(p) for p in k.pools]
        for w in want:
            w[spare] = w[int(k.table[0, 0])]
        new = D.accept(want, [k.table] * 2, [0, 0], k.ctx, k.off, k.path, k.len, [2, 2], [64, 64])
        g.replay()
        torch.cuda.synchronize()
        for p, w in zip(k.pools, want):
            np.testing.assert_array_equal(D.bits(p), w)
        np.testing.assert_array_equal(k.batch.ctx_lens.cpu().numpy(), new)
