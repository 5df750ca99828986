"""The operators of a speculative step in the order a serving program uses them: forks of a prompt found as groups, a block
whose heads are normalised run over their drafted trees with the prefix read once, the trees verified on the target's
probabilities, the accepted paths kept, and on. A second program does the same steps with every sequence by itself, one
verified token at a time."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D
import serve_ref as S
import workloads as W
from harness import f64, rel_err
from workloads import gen

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402

PAGE, H, VOCAB = 16, 512, 777
CFGS = [W.LayerCfg(hidden=H, n_q=8, n_kv=2, head_dim=64, ffn=640), W.LayerCfg(hidden=H, n_q=8, n_kv=2, head_dim=64, ffn=640, window=200)]
TOL = 1e-2  # normwise per row, as the decode steps against the oracle: both sides run the same bf16 layers


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("axes", [False, True])
def test_fork_draft_verify_keep(axes):
    print("[case] serving", axes, file=sys.stderr, flush=True)
    rng = np.random.default_rng(4 + axes)
    P, rows, prompt = 160, 5, 150
    weights = [{k: v.cuda() for k, v in gen.layer_weights(c, 3, l, "cpu", H ** -0.5).items()} for l, c in enumerate(CFGS)]
    gains = [torch.from_numpy(1 + 0.2 * rng.standard_normal(64)).to(torch.bfloat16).cuda() for _ in range(4)]
    norm = [R.HeadNorm(gains[2 * l], gains[2 * l + 1]) for l in range(2)]
    # a rope of several axes turns rows of text as one of a single axis does: every axis is at the token's position
    rope = [R.Rope(64, rotary_dim=48, sections=(4, 10, 10), order="cyclic") if axes else R.Rope(64)] * 2
    embed = torch.from_numpy(rng.standard_normal((VOCAB, H)).astype(np.float32)).to(torch.bfloat16).cuda()
    head = torch.from_numpy(rng.standard_normal((H, VOCAB)).astype(np.float32) * 0.15).cuda()
    pools = [gen.kv_pool(c, P, 5, l, "cpu").cuda() for l, c in enumerate(CFGS)]
    block = R.DeviceBlock(CFGS, weights, pools, P)
    k = R.KvPages(P, rows + 3, 24)
    k.resize(0, prompt)                         # the pool's random contents stand for the prompt's cache
    for b in (1, 2, 3):
        k.fork(0, b)
    k.resize(4, 21)                             # one with a prompt of its own
    for b, src in ((5, 0), (6, 1), (7, 4)):     # the plain program's sequences
        k.fork(src, b)

    def copies():
        for c in k.take_copies():
            R.kv_copy_pages(block, cuda(c))

    def step(seqs, tokens, counts, depth, sets, max_rows, shared):
        """Logits of every row; ctx counts the cached tokens."""
        ctx = k.tokens[seqs].copy()
        for b, n in zip(seqs, counts):
            k.resize(b, int(k.tokens[b]) + n)
        copies()
        off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        table = np.full((len(seqs), 4096 if shared else k.table.shape[1]), -1, np.int32)  # groups are taken by tables that span 128 MB
        table[:, :k.table.shape[1]] = k.table[seqs]
        batch = R.DeviceBatch(cuda(ctx), cuda(table))
        draft = R.DeviceDraft(cuda(off), cuda(np.asarray(depth, np.int32)), cuda(D.mask_words(sets, max_rows)), max_rows=max_rows,
                              rope=rope, norm=norm, shared=shared)
        state = R.DeviceState(block, batch, fill=float("nan"), draft=draft)
        x = state.view("resid", int(off[-1]), H)
        x.copy_(embed[cuda(np.asarray(tokens, np.int64))])
        R.run_draft(block, 0, block.num_ops(), batch, draft, state)
        return x.clone(), batch, draft, off, ctx

    last = [3, 3, 3, 3, 7]                      # the token each sequence ended with
    verifier = R.DraftVerifier(rows, 9, VOCAB)
    kept_all = [[] for _ in range(rows)]
    for it in range(3):
        counts = [int(n) for n in rng.integers(1, 9, rows)]
        depth, sets, parent, tokens = [], [], [], []
        for b, n in enumerate(counts):
            up = [-1] + [max(0, j - 1 - int(rng.integers(0, 3))) for j in range(1, n)]
            d, anc = [0], [[0]]
            for j in range(1, n):
                d.append(d[up[j]] + 1)
                anc.append(anc[up[j]] + [j])
            depth, sets, parent = depth + d, sets + anc, parent + up
            tokens += [last[b]] + [int(t) for t in rng.integers(0, VOCAB, n - 1)]
        off_g, claims = k.shared()
        at = [i for i, o in enumerate(off_g.tolist()) if o <= rows]
        groups = R.SharedPrefix(cuda(np.minimum(off_g[:len(at) + 1], rows)[:len(at)].astype(np.int32)), cuda(claims[:len(at) - 1]))
        assert claims[0] >= prompt // PAGE * PAGE and off_g[1] == 4
        out, batch, draft, off, ctx = step(list(range(rows)), tokens, counts, depth, sets, max(counts), groups)
        target = torch.softmax(out.float() @ head, dim=1)
        # drafts the target likes, so that paths grow: every second child is its parent's likeliest token. Tokens are inputs
        # of the step, so it is run again with them (the same slots; what the rows see does not depend on later rows).
        for b in range(rows):
            for j in range(1, counts[b]):
                if j % 2:
                    tokens[off[b] + j] = int(target[off[b] + parent[off[b] + j]].argmax())
            k.resize(b, int(ctx[b]))
        out, batch, draft, off, ctx = step(list(range(rows)), tokens, counts, depth, sets, max(counts), groups)
        target = torch.softmax(out.float() @ head, dim=1)
        u = rng.random(len(tokens)).astype(np.float32) * 0.3
        v = rng.random(rows).astype(np.float32)
        verifier.run(draft, cuda(np.array(tokens, np.int32)), cuda(np.array(parent, np.int32)), target, cuda(u), cuda(v))
        R.kv_accept(block, batch, draft, verifier.path, verifier.path_len, ctx_out=batch.ctx_lens)
        torch.cuda.synchronize()
        path, lens, nxt = S.verify(off, len(tokens), max(counts), tokens, parent, f64(target), None, u, v, 9, VOCAB)
        np.testing.assert_array_equal(verifier.path.cpu().numpy(), path)
        np.testing.assert_array_equal(verifier.next.cpu().numpy(), nxt)
        np.testing.assert_array_equal(batch.ctx_lens.cpu().numpy(), ctx + lens)

        # the plain program: the kept tokens one at a time, each sequence by itself
        for slow, b in ((5, 0), (6, 1), (7, 4)):
            for i in range(int(lens[b])):
                row = int(off[b] + path[b, i])
                ref = step([slow], [tokens[row]], [1], [0], [[0]], 1, None)[0]
                e = rel_err(f64(out[row]), f64(ref[0]))
                assert e <= TOL, f"step {it}, sequence {b}, kept row {i}: {e}"
        for b in range(rows):
            k.resize(b, int(ctx[b]) + int(lens[b]))
            kept_all[b].append(int(lens[b]))
            last[b] = int(nxt[b])
        copies()
    assert max(max(x) for x in kept_all) > 1
    for b in range(rows + 3):
        k.release(b)
    assert k.free == P
