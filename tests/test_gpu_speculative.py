"""The operators in the order a serving program uses them: fork two continuations of a prompt, run their drafted trees
through a whole block, keep one path of each, give back what is not needed, compact the pool, decode on. Every step is
compared with plain decode steps of the same tokens on a cache of their own."""
import sys
from dataclasses import replace

import numpy as np
import pytest
import torch

import draft_ref as D
import workloads as W
from harness import f64, rel_err
from workloads import gen

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402

PAGE = 16
BASE = W.LayerCfg(hidden=512, n_q=8, n_kv=2, head_dim=64, ffn=640)
TOL = 1e-2  # normwise per row, as the decode steps against the oracle: both sides run the same bf16 layers


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Model:
    """Two layers, weights, and a decode step of given residual rows at given contexts over given pools."""

    def __init__(self, cfgs, P, seed, rope):
        self.cfgs, self.P, self.rope = cfgs, P, rope
        self.weights = [{k: v.cuda() for k, v in gen.layer_weights(c, seed, l, "cpu", 512 ** -0.5).items()}
                        for l, c in enumerate(cfgs)]
        self.n_ops = sum(c.n_ops for c in cfgs)

    def block(self, pools):
        return R.DeviceBlock(self.cfgs, self.weights, pools, self.P)

    def drafted(self, block, ctx, table, x, counts, depth, sets, max_rows):
        """One step over drafted rows: the residual rows out."""
        off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        batch = R.DeviceBatch(cuda(np.asarray(ctx, np.int32)), cuda(table))
        draft = R.DeviceDraft(cuda(off), cuda(np.asarray(depth, np.int32)), cuda(D.mask_words(sets, max_rows)), max_rows=max_rows,
                              rope=None if self.rope is None else [self.rope] * len(self.cfgs))
        state = R.DeviceState(block, batch, fill=float("nan"), draft=draft)
        state.view("resid", len(x), self.cfgs[0].hidden).copy_(x)
        R.run_draft(block, 0, self.n_ops, batch, draft, state)
        return state.view("resid", len(x), self.cfgs[0].hidden).clone(), batch, draft

    def decode(self, block, ctx, table, x):
        """One plain decode step: ctx tokens with the new one. A rope of its own takes the drafted form, a row each."""
        if self.rope is not None:
            B = len(ctx)
            return self.drafted(block, np.asarray(ctx) - 1, table, x, [1] * B, [0] * B, [[0]] * B, 1)[0]
        batch = R.DeviceBatch(cuda(np.asarray(ctx, np.int32)), cuda(table))
        state = R.DeviceState(block, batch, fill=float("nan"))
        state.view("resid", len(x), self.cfgs[0].hidden).copy_(x)
        R.run_partition(block, 0, self.n_ops, batch, state)
        return state.view("resid", len(x), self.cfgs[0].hidden).clone()


@pytest.mark.parametrize("kind", ["own rope", "scaled rope", "window", "moe"])
def test_draft_verify_keep_and_decode(kind):
    print("[case] speculative", kind, file=sys.stderr, flush=True)
    cfgs = [BASE, BASE]
    if kind == "window":
        cfgs = [replace(BASE, window=40), BASE]
    elif kind == "moe":
        cfgs = [BASE, replace(BASE, ffn=0, n_experts=8, top_k=8, moe_ffn=128)]   # every expert: no near-ties between runs
    rope = R.Rope(64, rotary_dim=48, interleaved=True, scaling="index", factor=4.0, orig_ctx=64) if kind == "scaled rope" else None
    P, rows, max_pages = 64, 4, 12
    m = Model(cfgs, P, 3, rope)
    rng = np.random.default_rng(2)
    hidden = lambda n: torch.from_numpy(rng.standard_normal((n, 512)).astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
    pools = [gen.kv_pool(c, P, 5, l, "cpu").cuda() for l, c in enumerate(cfgs)]
    block = m.block(pools)

    k = R.KvPages(P, rows, max_pages)
    prompt = 37
    k.resize(0, prompt)                     # the pool's random contents stand for the prompt's cache
    k.fork(0, 1)
    k.fork(0, 2)                            # the plain reference's two sequences
    k.fork(0, 3)
    n = [11, 20]
    for b in (0, 1):
        k.resize(b, prompt + n[b])
    for b in (2, 3):
        k.resize(b, prompt + 12)

    def copies():
        for c in k.take_copies():
            R.kv_copy_pages(block, cuda(c))

    copies()
    trees = [D.forest(x, rng) for x in n]
    x = hidden(sum(n))
    out, batch, draft = m.drafted(block, [prompt] * 2, k.table[:2], x, n, trees[0][0] + trees[1][0],
                                  trees[0][1] + trees[1][1], max(n))
    paths = [max(t[1], key=len) for t in trees]
    paths[0] = paths[0][:-1] if len(paths[0]) > 2 else paths[0]
    width = max(map(len, paths))
    path = np.zeros((2, width), np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    lens = np.array([len(p) for p in paths], np.int32)
    R.kv_accept(block, batch, draft, cuda(path), cuda(lens), ctx_out=batch.ctx_lens)
    torch.cuda.synchronize()
    assert batch.ctx_lens.tolist() == [prompt + len(p) for p in paths]

    # plain decode steps of the kept tokens, one at a time, on rows 2 and 3
    worst = 0.0
    for step in range(width):
        live = [b for b in (0, 1) if step < len(paths[b])]
        at = [sum(n[:b]) + paths[b][step] for b in live]
        ref = m.decode(block, [prompt + step + 1 for _ in live], k.table[[2 + b for b in live]], x[at])
        for i, r in enumerate(at):
            e = rel_err(f64(out[r]), f64(ref[i]))
            assert e <= TOL, f"row {r} (step {step}): {e}"
            worst = max(worst, e)
    for b in (0, 1):
        k.resize(b, prompt + len(paths[b]))
        k.resize(2 + b, prompt + len(paths[b]))
    copies()

    # the caches agree slot by slot
    for c, pool in zip(cfgs, pools):
        hp = pool.double().cpu().numpy()
        for b in (0, 1):
            for t in range(prompt + len(paths[b])):
                for g, w in zip(D.slot(hp, k.table[b], t, 0, c.n_kv, 64), D.slot(hp, k.table[2 + b], t, 0, c.n_kv, 64)):
                    assert np.abs(g - w).max() <= TOL * max(1.0, np.abs(w).max()), (b, t)

    # compaction moves pages and nothing else; two more tokens decode alike on both
    moved = k.compact()
    assert k.table.max() < P - k.free
    copies()
    for step in range(2):
        for b in range(4):
            k.resize(b, int(k.tokens[b]) + 1)
        copies()
        y = hidden(2)
        got = m.decode(block, [int(t) for t in k.tokens], k.table, torch.cat([y, y]))
        torch.cuda.synchronize()
        for b in (0, 1):
            e = rel_err(f64(got[b]), f64(got[2 + b]))
            assert e <= TOL, f"after compaction ({moved} moved), sequence {b}, step {step}: {e}"
    for b in range(4):
        k.release(b)
    assert k.free == P


def test_tensors_off_the_current_device_are_refused():
    """Host tensors stand in for another device's: the check is the same."""
    r = R.Rope(64)
    x, pos = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for a, b, out in ((x, pos, None), (x.cuda(), pos, None), (x, pos.cuda(), None), (x.cuda(), pos.cuda(), x)):
        with pytest.raises(ValueError, match="current device"):
            R.rope(r, a, b, out=out)
    with pytest.raises(ValueError, match="current device"):
        R.rope(R.Rope(64, device="cpu"), x.cuda(), pos.cuda())
    cfg = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)
    pool = torch.zeros(8, 2, 2, 16 * 64, dtype=torch.bfloat16, device="cuda")
    block = R.DeviceBlock([cfg], [{}], [pool], 8)
    ints = lambda *v, **kw: torch.tensor(v, dtype=torch.int32, **kw)  # noqa: E731
    with pytest.raises(ValueError, match="current device"):
        R.kv_copy_pages(block, ints(0, 1).reshape(1, 2))
    with pytest.raises(ValueError, match="contiguous"):
        R.kv_copy_pages(block, torch.zeros(4, 2, dtype=torch.int32, device="cuda")[:, :1].expand(4, 2))
    batch = R.DeviceBatch(ints(3, device="cuda"), ints(0, 1, device="cuda").reshape(1, 2))
    draft = R.DeviceDraft(ints(0, 2), ints(0, 1), torch.ones(2, dtype=torch.int64), max_rows=2)
    state = R.DeviceState(block, batch, draft=draft)
    with pytest.raises(ValueError, match="current device"):
        R.run_draft(block, 4, 5, batch, draft, state)
    with pytest.raises(ValueError, match="current device"):
        R.kv_accept(block, batch, draft, ints(0, 1).reshape(1, 2), ints(1))
