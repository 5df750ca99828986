"""Attention of drafted rows whose sequences share a prefix (ods_draft.shared) against the definition in 64 bits over each
sequence's own table: groups of every size, prefixes around tiles and pages, lengths from one token, trees, what is not
finite, tables that end, captured graphs whose groups change, many groups and launches."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D
import workloads as W

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402
from test_gpu_tree import Case  # noqa: E402

PAGE = 16
SPAN = 128 << 20


def say(*a):
    print("[case] shared", *a, file=sys.stderr, flush=True)


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Shared(Case):
    """groups: (sequences, shared tokens, claimed tokens or None). The tables of a group name the same pages for its whole
    shared pages; ctx counts from the front as ever."""

    def __init__(self, groups, ctx, rows, **kw):
        super().__init__(ctx, rows, **kw)
        self.group_off = np.concatenate([[0], np.cumsum([g[0] for g in groups])]).astype(np.int32)
        self.tokens = np.array([g[1] if len(g) < 3 else g[2] for g in groups], np.int32)
        b = 0
        for g in groups:
            self.table[b:b + g[0], :g[1] // PAGE] = self.table[b, :g[1] // PAGE]
            b += g[0]

    def device(self, rope=None, shared=True, more=False):
        """Groups are taken where the tables span 128 MB: of more columns, or (`more`) of more sequences, which are left alone."""
        super().device(rope)
        self.prefix = R.SharedPrefix(cuda(self.group_off), cuda(self.tokens))
        if shared:
            B, cols = self.table.shape
            least = SPAN // (PAGE * self.n_kv * self.hd * 4)
            wide = np.full((max(B, -(-least // cols)), cols) if more else (B, max(cols, -(-least // B))), -1, np.int32)
            wide[:B, :cols] = self.table
            ctx, off = np.full(len(wide), -1, np.int32), np.full(len(wide) + 1, self.off[-1], np.int32)
            ctx[:B], off[:B] = self.ctx, self.off[:B]
            self.batch = R.DeviceBatch(cuda(ctx), cuda(wide), ring_table=None)
            self.draft = R.DeviceDraft(cuda(off), cuda(self.depth), cuda(D.mask_words(self.sets, self.max_rows)),
                                       max_rows=self.max_rows, rope=rope, shared=self.prefix)
            self.state = R.DeviceState(self.block, self.batch, fill=float("nan"), draft=self.draft)
            self.state.view("qkv", *self.qkv.shape).copy_(self.qkv)
            self.state.view("o", self.R, self.n_q * self.hd).fill_(-3.0)
        return self


HEADS = [(4, 2, 64), (8, 1, 64), (16, 1, 128), (8, 2, 128), (3, 3, 128), (6, 2, 64)]


@pytest.mark.parametrize("n_q,n_kv,hd", HEADS)
@pytest.mark.parametrize("members", [2, 3, 17, 70])
def test_single_tokens_of_groups_of_every_size(n_q, n_kv, hd, members):
    say("members", n_q, n_kv, hd, members)
    rng = np.random.default_rng(members)
    ctx = 96 + rng.integers(0, 120, members)
    c = Shared([(members, 96)], ctx, [1] * members, n_q=n_q, n_kv=n_kv, hd=hd, seed=members).device()
    c.check(c.attend())


@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 31, 32, 33, 47, 48, 64, 95, 500, 1000])
@pytest.mark.parametrize("hd", [64, 128])
def test_prefixes_around_pages_and_tiles(prefix, hd):
    """Only whole tiles of the shared pages are read once. Contexts end with the prefix, a token later, or much later."""
    say("prefix", prefix, hd)
    whole = prefix // PAGE * PAGE
    ctx = [whole, whole + 1, whole + 17, whole + 200, whole + 31]
    c = Shared([(5, whole)], ctx, [3, 1, 7, 2, 1], n_q=8, n_kv=2, hd=hd, seed=prefix).device()
    c.check(c.attend())


@pytest.mark.parametrize("n", [1, 2, 3, 5, 8, 9, 16, 32, 33, 64])
@pytest.mark.parametrize("group,hd", [(1, 64), (4, 128), (16, 64)])
def test_trees_of_every_width(n, group, hd):
    say("width", n, group, hd)
    ctx = [200, 233, 192, 700, 64, 70, 80, 81]
    c = Shared([(4, 192), (4, 64)], ctx, [n] * 8, n_q=2 * group, n_kv=2, hd=hd, seed=n).device()
    c.check(c.attend())


@pytest.mark.parametrize("n_q,n_kv,hd,n", [(16, 1, 64, 2), (8, 2, 64, 5), (16, 1, 128, 1), (8, 2, 128, 8), (3, 3, 128, 32)])
def test_groups_of_a_thousand_columns(n_q, n_kv, hd, n):
    say("columns", n_q, n_kv, hd, n)
    members = 80
    ctx = 160 + np.arange(members) * 3
    rows = [n - b % 2 for b in range(members)] if n > 1 else [1] * members
    c = Shared([(members, 160)], ctx, rows, n_q=n_q, n_kv=n_kv, hd=hd, seed=n, max_rows=n).device()
    c.check(c.attend())


def test_ragged_groups_with_everything_in_them():
    """Groups of one, of none, sequences in no group on both sides, one left alone, one without rows, rows past the most,
    contexts shorter than the group's prefix, padding rows."""
    say("ragged")
    ctx = [40, 400, 401, 415, -1, 390, 100, 3, 64, 0, 1000, 1200, 1024, 77, 9]
    rows = [3, 2, 0, 12, 2, 5, 4, 1, 6, 3, 1, 8, 2, 1, 4]
    c = Shared([(0, 0), (7, 384), (2, 0), (1, 0), (3, 992)], ctx, rows, n_q=8, n_kv=2, hd=128, seed=1, max_rows=8, pad=6)
    c.group_off = np.array([1, 1, 8, 10, 10, 13], np.int32)   # sequences 0, 13 and 14 in no group
    c.tokens = np.array([50, 384, 0, 64, 992], np.int32)
    for a, e, k in ((1, 8, 384), (10, 13, 992)):
        c.table[a:e, :k // PAGE] = c.table[a, :k // PAGE]
    c.device()
    c.check(c.attend())


@pytest.mark.parametrize("max_rows", [65, 128, 256])
def test_masks_of_several_words(max_rows):
    """More columns than groups are taken for."""
    say("words", max_rows)
    c = Shared([(3, 320)], [320, 340, 700], [max_rows, 66, 1], n_q=4, n_kv=2, hd=64, seed=max_rows, max_rows=max_rows).device()
    c.check(c.attend())


def test_long_prefixes_cut_into_many_ranges():
    say("long")
    for members, rows, n_q, n_kv, hd in ((2, 1, 4, 1, 64), (40, 2, 32, 8, 128), (6, 2, 16, 1, 128)):
        ctx = 9000 + np.arange(members) * 37
        c = Shared([(members, 8992)], ctx, [rows] * members, n_q=n_q, n_kv=n_kv, hd=hd, seed=members).device()
        c.check(c.attend())


@pytest.mark.parametrize("hd,n,tail", [(128, 4, 700), (128, 2, 700), (64, 4, 1400)])
def test_long_ranges_of_whole_tails(hd, n, tail):
    """Ranges of one wave that pass several tails and more than 32 tiles, beside a prefix long enough to leave them few
    compute units. The definition is computed on the GPU in 64 bits."""
    say("long tails", hd, n, tail)
    B, g, prefix = 128, 8, 65536
    rng = np.random.default_rng(hd + n)
    ctx = prefix + rng.integers(tail // 3, tail, B)
    own = -(-(ctx + n) // PAGE) - prefix // PAGE
    P = prefix // PAGE + int(own.sum())
    ids, at = rng.permutation(P).astype(np.int32), prefix // PAGE
    table = np.full((B, prefix // PAGE + int(own.max())), -1, np.int32)
    table[:, :prefix // PAGE] = ids[:prefix // PAGE]
    for b, k in enumerate(own):
        table[b, prefix // PAGE:prefix // PAGE + k] = ids[at:at + k]
        at += k
    gen = torch.Generator(device="cuda").manual_seed(hd)
    pool = torch.randn((P, 2, 1, PAGE * hd), generator=gen, device="cuda").to(torch.bfloat16)
    qkv = torch.randn((B * n, (g + 2) * hd), generator=gen, device="cuda").to(torch.bfloat16)
    block = R.DeviceBlock([W.LayerCfg(hidden=256, n_q=g, n_kv=1, head_dim=hd, ffn=512)], [{}], [pool], P)
    batch = R.DeviceBatch(cuda(ctx.astype(np.int32)), cuda(table))
    draft = R.DeviceDraft(cuda(np.arange(B + 1, dtype=np.int32) * n), cuda(np.tile(np.arange(n, dtype=np.int32), B)),
                          cuda(np.tile((2 << np.arange(n)) - 1, B).astype(np.int64)), max_rows=n,
                          shared=R.SharedPrefix(cuda(np.array([0, B], np.int32)), cuda(np.array([prefix], np.int32))))
    state = R.DeviceState(block, batch, fill=float("nan"), draft=draft)
    state.view("qkv", *qkv.shape).copy_(qkv)
    R.run_draft(block, 4, 5, batch, draft, state)
    torch.cuda.synchronize()
    got = state.view("o", B * n, g * hd).double().cpu().numpy().reshape(B, n, g, hd)
    for b in range(B):
        last = int(ctx[b]) + n
        pages = pool[torch.from_numpy(table[b, :-(-last // PAGE)].astype(np.int64)).cuda()].double()
        k = pages[:, 0, 0].reshape(-1, hd)[:last]
        v = pages[:, 1, 0].view(-1, hd, PAGE).transpose(1, 2).reshape(-1, hd)[:last]
        s = qkv[b * n:(b + 1) * n, :g * hd].double().reshape(n * g, hd) @ k.T / hd ** 0.5
        s = s.view(n, g, last)
        for j in range(n):
            s[j, :, int(ctx[b]) + j + 1:] = -float("inf")   # a chain: rows see those before them
        p = torch.softmax(s, dim=2).view(n * g, last)
        o, mag = ((p @ x).cpu().numpy().reshape(n, g, hd) for x in (v, v.abs()))
        off = np.abs(got[b] - o) - D.tree_bound(o, mag)
        assert (off <= 0).all(), f"sequence {b}: off by {off.max()} more than the bound"


def test_hidden_rows_and_what_is_not_finite():
    """A drafted row of no mask bit attends the cache alone. Infinities and NaN in pages behind a sequence's tokens, in
    slots past its end and in drafted rows it may not see do not reach it; in the prefix they reach every row."""
    say("non-finite")
    ctx, rows = [130, 140, 128, 300], [6, 3, 1, 2]
    c = Shared([(3, 128), (1, 0)], ctx, rows, n_q=8, n_kv=2, hd=64, seed=3)
    c.sets[1], c.sets[4] = [], [0]
    for b in range(4):
        for p in range(-(-(ctx[b] + rows[b]) // PAGE), c.table.shape[1]):
            c.pool[c.table[b, p]] = float("nan")
    last = c.table[0, (130 + 5) // PAGE]
    c.pool[last].view(2, 2, PAGE * 64)[1].view(2, 64, PAGE)[..., (130 + 5) % PAGE] = float("inf")   # value of drafted row 5
    c.device()
    c.check(c.attend())
    o = c.o().clone()
    c.pool[c.table[0, 2]].view(2, 2, PAGE * 64)[1].view(2, 64, PAGE)[0, 7, 3] = float("inf")       # dim 7 of a shared token
    c.device()
    got = c.attend()
    c.check(got)
    bad = ~torch.isfinite(got[:10].view(10, 8, 64)[:, :4])
    assert bad[..., 7].all() and torch.equal(got[10:], o[10:])


def test_pages_outside_the_pool_and_tables_that_end():
    say("bad pages")
    ctx = [200, 210, 230, 256, 250]
    c = Shared([(4, 192), (1, 0)], ctx, [2, 16, 1, 9, 16], n_q=4, n_kv=2, hd=64, seed=5)
    c.table[:4, 3], c.table[:4, 4], c.table[1, 12] = -1, c.P + 5, -7
    c.table = c.table[:, :16].copy()                # 256 tokens: what does not fit is neither written nor attended
    c.device(more=True)
    c.check(c.attend())
    c = Shared([(3, 64)], [64, 64, 64], [4, 1, 2], n_q=4, n_kv=2, hd=128, seed=6)
    c.table = c.table[:, :4].copy()                 # a prefix as wide as the table: its last tile is each one's own
    c.device(more=True)
    c.check(c.attend())


def test_claims_that_pass_the_table_or_are_negative():
    say("claims")
    for claim in (-5, 2 ** 31 - 1, 10_000):
        for more in (False, True):
            c = Shared([(3, 160, claim)], [170, 180, 176], [2, 1, 3], n_q=4, n_kv=2, hd=64, seed=7).device(more=more)
            c.check(c.attend())


def test_offsets_that_do_not_ascend_share_nothing():
    """Device arrays that break their contract are computed without a prefix (offsets that descend, or outside the batch), or
    at least stay inside the buffers (rows that do not ascend)."""
    say("offsets")
    ctx = [200 + 7 * b for b in range(8)]
    for off in ([0, 8, 0, 8, 0, 8], [5, 4, 3, 2, 1, 0], [-2 ** 31, 2 ** 31 - 1, -1, 3, 9, 8], [8, 8, 8, 2 ** 31 - 1, 9, 0]):
        c = Shared([(8, 192)], ctx, [3] * 8, n_q=8, n_kv=2, hd=64, seed=14)
        c.group_off, c.tokens = np.array(off, np.int64).astype(np.int32), np.full(5, 192, np.int32)
        c.device()
        c.check(c.attend())
    for off in ([-7, 3, 3, 8], [0, 4, 2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, -2 ** 31, 0, 100]):   # clipped to the batch
        c = Shared([(8, 192)], ctx, [3] * 8, n_q=8, n_kv=2, hd=64, seed=15)
        c.group_off, c.tokens = np.array(off, np.int64).astype(np.int32), np.full(3, 192, np.int32)
        c.device()
        c.check(c.attend())
    c = Shared([(4, 192), (4, 192)], ctx, [3] * 8, n_q=8, n_kv=2, hd=64, seed=16).device()
    c.draft.row_off.copy_(cuda(np.array([0, 24, 3, 24, 9, 12, 24, 18, 24], np.int32)))
    c.attend()   # no more than that it ends


def test_sliding_window_layers_read_their_own_windows():
    say("window")
    c = Shared([(4, 320)], [330, 350, 320, 400], [3, 2, 1, 5], n_q=4, n_kv=2, hd=64, window=50, seed=8).device()
    got = c.attend()
    c.check(got)
    c.device(shared=False)
    assert torch.equal(got, c.attend())


def test_many_groups_and_batches_of_several_launches():
    say("many")
    rng = np.random.default_rng(9)
    for B, size in ((1024, 2), (4096, 9), (1500, 3)):
        groups = [(size, 32)] * (B // size)  # the last sequences may be in no group
        ctx = 32 + rng.integers(0, 20, B)
        c = Shared(groups, ctx, rng.integers(0, 3, B), n_q=2, n_kv=1, hd=64, seed=B, max_rows=2).device()
        got = c.attend()
        c.device(shared=False)
        plain = c.attend()
        # both are within the bound of the 64-bit ones (the batch is too large to compute those here): twice half a bf16
        # step of each, and of the probabilities
        d, most = (got.float() - plain.float()).abs(), float(c.pool.abs().max())
        assert (d <= 2 * 2.0 ** -8 * (plain.float().abs().maximum(got.float().abs()) + 33 / 32 * most)).all()
    sub = Shared([(4, 32)] * 512, 32 + rng.integers(0, 9, 2048), [1] * 2048, n_q=2, n_kv=1, hd=64, seed=3)
    sub.device()
    sub.check(sub.attend())


def test_captured_graph_whose_groups_change():
    """Contexts, rows, groups and prefixes of a captured call change between replays; eager work between them."""
    say("graph")
    c = Shared([(4, 320), (4, 0)], [330, 350, 320, 400, 40, 50, 60, 300], [3, 2, 1, 5, 2, 2, 2, 2], n_q=8, n_kv=2, hd=128, seed=10).device()
    g = R.DraftGraph(c.block, 4, 5, c.batch, c.draft, c.state)
    for bounds, tokens in (((0, 4, 8), (320, 0)), ((0, 2, 4), (320, 64)), ((0, 0, 4), (7, 300)), ((0, 8, 8), (0, 0)), ((0, 4, 8), (320, 0))):
        c.prefix.group_off.copy_(cuda(np.array(bounds, np.int32)))
        c.prefix.tokens.copy_(cuda(np.array(tokens, np.int32)))
        c.ctx[:4] += 1
        c.ctx[4:] += 3
        c.batch.ctx_lens.copy_(cuda(c.ctx))
        c.o().fill_(-3.0)
        g.launch()
        torch.cuda.synchronize()
        got = c.o().clone()
        c.check(got)
        c.o().fill_(-3.0)
        assert torch.equal(c.attend(), got)
    g.close()


def test_sequences_that_end_between_calls():
    """What an earlier call left in the workspace is not joined for sequences that are left alone now, of any KV head."""
    say("left alone")
    c = Shared([(3, 96)], [100, 130, 96], [2, 1, 2], n_q=300, n_kv=300, hd=64, seed=17).device()
    c.check(c.attend())
    c.ctx[1] = -1
    c.batch.ctx_lens.copy_(cuda(c.ctx))
    got = c.attend()
    c.check(got)
    assert (got[2] == 0).all()


def test_the_same_twice_and_on_another_stream():
    say("stream")
    c = Shared([(40, 2000)], 2000 + np.arange(40) * 11, [2] * 40, n_q=32, n_kv=8, hd=128, seed=11).device()
    first = c.attend()
    assert torch.equal(first, c.attend())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.o().fill_(-3.0)
        R.run_draft(c.block, 4, 5, c.batch, c.draft, c.state)
    torch.cuda.synchronize()
    assert torch.equal(first, c.o())


def test_groups_found_by_the_page_bookkeeping():
    say("pages")
    k = R.KvPages(pool_pages=400, rows=7, max_pages=40)
    k.resize(0, 321)
    for b in (1, 2):
        k.fork(0, b)
    k.resize(3, 50)
    k.resize(4, 160)
    for b in (5, 6):
        k.fork(4, b)
    for b, n in enumerate([330, 400, 325, 60, 161, 170, 300]):
        k.resize(b, n)
    off, tokens = k.shared()
    assert off.tolist() == [0, 3, 4, 7] and tokens.tolist() == [320, 0, 160]
    c = Shared([(7, 0)], k.tokens, [2, 1, 3, 1, 2, 2, 1], n_q=4, n_kv=2, hd=64, seed=12)
    for b, n in enumerate(c.n):
        k.resize(b, int(c.ctx[b]) + int(n))
    c.P = 400
    c.pool = torch.from_numpy(np.random.default_rng(0).standard_normal((400, 2, 2, PAGE * 64)).astype(np.float32)).to(torch.bfloat16)
    c.table, c.group_off, c.tokens = k.table.copy(), off, tokens
    c.device()
    c.check(c.attend())


def test_a_state_for_the_widest_serves_narrower_drafts():
    say("state")
    wide = Shared([(6, 640)], [640 + 9 * i for i in range(6)], [32] * 6, n_q=16, n_kv=2, hd=128, seed=13).device()
    wide.check(wide.attend())
    state = wide.state
    for n in (1, 2, 3, 4, 5, 16, 31):
        c = Shared([(3, 640), (2, 0)], [650 + i for i in range(5)], [n] * 5, n_q=16, n_kv=2, hd=128, seed=n).device()
        assert c.state.ws_bytes <= state.ws_bytes
        state.view("qkv", *c.qkv.shape).copy_(c.qkv)
        state.view("o", c.R, c.n_q * c.hd).fill_(-3.0)
        R.run_draft(c.block, 4, 5, c.batch, c.draft, state)
        torch.cuda.synchronize()
        c.check(state.view("o", c.R, c.n_q * c.hd).clone())
