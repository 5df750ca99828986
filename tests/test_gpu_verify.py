"""Verification of drafted tokens (ods_draft_verify) against its definition, token by token in 64 bits: chains and trees,
with and without the draft's probabilities, vocabularies around the chunks, strides, types, what is not a probability."""
import sys

import numpy as np
import pytest
import torch

import serve_ref as S

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402


def say(*a):
    print("[case] verify", *a, file=sys.stderr, flush=True)


def t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Case:
    def __init__(self, counts, vocab, spread, drawn, seed=0, dtype=torch.float32, pad=0, lead=0, max_rows=None, path_cols=None,
                 sharp=2.0, padding_rows=0):
        rng = self.rng = np.random.default_rng(seed)
        self.off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        rows = self.rows = int(self.off[-1]) + padding_rows
        self.vocab = vocab
        self.max_rows = max(1, max(counts)) if max_rows is None else max_rows
        self.path_cols = self.max_rows if path_cols is None else path_cols
        self.parent = np.full(rows, -1, np.int32)
        logits = sharp * rng.standard_normal((rows, vocab))
        blur = 0.8 * logits + 0.6 * rng.standard_normal((rows, vocab))
        soft = lambda z: np.exp(z - z.max(1, keepdims=True)) / np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)  # noqa: E731
        wide = lambda p: torch.from_numpy(np.pad(p.astype(np.float32), ((0, 0), (lead, pad)), constant_values=np.nan)).to(dtype).cuda()  # noqa: E731
        self.target = wide(soft(logits))[:, lead:lead + vocab]
        self.proposal = wide(soft(blur))[:, lead:lead + vocab] if drawn else None
        q = soft(blur)
        self.tokens = rng.integers(0, vocab, rows).astype(np.int32)
        for b in range(len(counts)):
            a = int(self.off[b])
            for j in range(1, counts[b]):
                p = max(0, j - 1 - int(rng.integers(0, spread)))
                self.parent[a + j] = p
                self.tokens[a + j] = rng.choice(vocab, p=q[a + p]) if drawn else rng.choice(np.argsort(-q[a + p])[:6])
        self.u = rng.random(rows).astype(np.float32)
        self.v = rng.random(len(counts)).astype(np.float32)

    def args(self):
        return t(self.tokens), t(self.parent), self.target, t(self.u), t(self.v)

    def draft(self):
        words = -(-self.max_rows // 64)
        return R.DeviceDraft(t(self.off), torch.zeros(self.rows, dtype=torch.int32, device="cuda"),
                             torch.zeros(self.rows, words, dtype=torch.int64, device="cuda"), max_rows=self.max_rows)

    def expect(self):
        f = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        return S.verify(self.off, self.rows, self.max_rows, self.tokens, self.parent, f(self.target), f(self.proposal), self.u,
                        self.v, self.path_cols, self.vocab)

    def check(self, verifier=None):
        B = len(self.off) - 1
        v = verifier or R.DraftVerifier(B, self.path_cols, self.vocab)
        v.run(self.draft(), *self.args(), proposal=self.proposal)
        torch.cuda.synchronize()
        path, lens, nxt = self.expect()
        np.testing.assert_array_equal(v.path_len[:B].cpu().numpy(), lens)
        np.testing.assert_array_equal(v.path[:B].cpu().numpy(), path)
        np.testing.assert_array_equal(v.next[:B].cpu().numpy(), nxt)
        return path, lens, nxt


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("spread", [1, 3])
@pytest.mark.parametrize("vocab", [1, 2, 15, 1000, 1023, 1024, 1025, 4097, 32000])
def test_vocabularies(vocab, spread, drawn):
    say("vocab", vocab, spread, drawn)
    lens = Case([8, 1, 5, 12], vocab, spread, drawn, seed=vocab).check()[1]
    assert (lens >= 1).all()


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("dtype,pad,lead", [(torch.float32, 3, 1), (torch.float32, 0, 0), (torch.bfloat16, 0, 0), (torch.bfloat16, 1, 0),
                                            (torch.bfloat16, 2, 3)])
def test_types_and_rows_that_start_anywhere(dtype, pad, lead, drawn):
    """NaN on both sides of every row: what is outside the vocabulary is not read into it."""
    say("strides", dtype, pad, lead, drawn)
    Case([6, 3, 9, 2, 4], 2051, 3, drawn, seed=pad + lead, dtype=dtype, pad=pad, lead=lead).check()


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("rows", [63, 64, 65, 130, 256])
def test_wide_trees(rows, drawn):
    """Many children of few rows: every one of them tested on what the ones before left."""
    say("wide", rows, drawn)
    c = Case([rows, 1, rows - 7], 300, 1, drawn, seed=rows)
    q = c.proposal if drawn else c.target
    for b in (0, 2):
        a, e = int(c.off[b]), int(c.off[b + 1])
        for j in range(1, e - a):
            up = 0 if j < rows // 2 else j // 2
            c.parent[a + j] = up
            if drawn:
                p = q[a + up].double().cpu().numpy()
                c.tokens[a + j] = c.rng.choice(300, p=p / p.sum())
    c.u[:] = np.minimum(c.u * 0.2 + 0.85, 0.9999)                    # most are refused
    path, lens, _ = c.check()
    assert lens[0] < 12


def test_rows_past_the_most_padding_and_sequences_without_rows():
    say("ragged")
    c = Case([3, 0, 9, 1, 0, 5], 700, 2, True, seed=2, max_rows=4, padding_rows=3)
    path, lens, nxt = c.check()
    assert lens[1] == 0 and nxt[1] == -1 and (path[1] == -1).all()
    c = Case([7] * 3, 700, 1, False, seed=3, path_cols=2)             # paths cut at two rows
    c.u[:] = 0.0
    path, lens, _ = c.check()
    assert (lens == 2).all()
    Case([7] * 3, 700, 1, True, seed=4, path_cols=256).check()
    Case([7] * 3, 700, 1, True, seed=5, path_cols=1).check()


def test_tokens_and_parents_that_are_none():
    say("bad rows")
    c = Case([9, 9], 500, 3, True, seed=6)
    c.tokens[2], c.tokens[4], c.parent[5], c.parent[6], c.parent[12] = 500, -1, 5, 8, -4
    c.check()
    c = Case([9, 9], 500, 3, False, seed=7)
    c.tokens[1], c.tokens[12], c.parent[3] = 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1
    c.check()


def test_borders():
    """Random numbers at the ends of [0, 1), equal probabilities, certain tokens, the same guess twice."""
    say("borders")
    for u, v in ((0.0, 0.0), (1 - 2.0 ** -24, 1 - 2.0 ** -24), (1 - 2.0 ** -24, 0.0)):
        for drawn in (False, True):
            c = Case([5, 5, 5], 1500, 2, drawn, seed=8)
            c.u[:], c.v[:] = u, v
            c.check()
            if drawn:
                c.proposal = c.target.clone()                        # p = q: everything is kept
                _, lens, _ = c.check()
            c.target = torch.zeros_like(c.target)
            c.target[:, 7] = 1.0
            c.tokens[:] = 7
            c.tokens[2] = 9
            c.proposal = c.target.clone() if drawn else None
            assert (c.check()[2] == 7).all()
            c.tokens[:] = 5                                          # every sibling the same token, of no probability
            assert (c.check()[2] == 7).all()
    c = Case([4], 2048, 1, False, seed=9)                            # equal powers of two: borders are exact
    c.target[:] = 2.0 ** -11
    for v in (0.0, 0.5, 0.25, 1 / 1024, 1 - 2.0 ** -24):
        c.v[:], c.u[:] = v, 2.0 ** -11                               # u = p is refused: 2047 tokens are left
        assert c.check()[2][0] == int(v * 2047) + (int(v * 2047) >= c.tokens[1])


def test_nothing_left_and_nothing_at_all():
    """Random numbers of 1 refuse even what is certain: then the target itself is drawn from; rows of zeros give -1."""
    say("nothing left")
    c = Case([3, 3, 3], 1100, 5, False, seed=10)
    c.target[:] = 0
    c.parent[[1, 2, 4, 5, 7, 8]] = 0
    c.target[0, 5], c.target[0, 1050] = 0.5, 0.5
    c.target[6, 1099] = 1e-30
    c.tokens[[1, 2, 4, 5, 7, 8]] = [5, 1050, 5, 6, 5, 6]
    c.u[:] = 1.0
    _, lens, nxt = c.check()
    assert (lens == 1).all() and nxt[0] in (5, 1050) and nxt[1] == -1 and nxt[2] == 1099
    c.target[6] = float("nan")
    assert c.check()[2][2] == -1


def test_what_is_no_probability_counts_as_zero():
    say("not finite")
    for drawn in (False, True):
        c = Case([6, 6], 1300, 2, drawn, seed=11)
        for x in (c.target, c.proposal):
            if x is not None:
                x[::2, 3::7] = float("nan")
                x[:, 5::11] = float("inf")
                x[1::3, 1::13] = -1.0
        c.check()


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab", [128000, 300007])
def test_large_vocabularies(vocab, drawn):
    say("large vocabulary", vocab, drawn)
    for seed in range(3):
        Case([4, 9], vocab, 3, drawn, seed=seed).check()


def test_large_batches_and_a_verifier_for_more():
    say("batch")
    rng = np.random.default_rng(1)
    v = R.DraftVerifier(4096, 6, 50)
    Case(rng.integers(0, 7, 4096).tolist(), 37, 3, True, seed=12, max_rows=6).check(v)
    Case(rng.integers(1, 7, 100).tolist(), 50, 3, False, seed=13, max_rows=6).check(v)


def test_no_rows_and_no_sequences():
    say("empty")
    for drawn in (False, True):
        v = R.DraftVerifier(5, 4, 40)
        v.path.fill_(-9), v.path_len.fill_(-9), v.next.fill_(-9)
        c = Case([0, 0, 0], 40, 1, drawn, seed=16, path_cols=4)
        v.run(c.draft(), *c.args(), proposal=c.proposal)
        torch.cuda.synchronize()
        assert (v.path[:3] == -1).all() and (v.path_len[:3] == 0).all() and (v.next[:3] == -1).all()
        assert (v.path[3:] == -9).all() and (v.path_len[3:] == -9).all() and (v.next[3:] == -9).all()
    c.off, c.v, before = c.off[:1], c.v[:0], v.path.clone()
    v.run(c.draft(), *c.args(), proposal=c.proposal)
    torch.cuda.synchronize()
    assert torch.equal(v.path, before)


def test_tokens_come_from_the_target():
    """4096 times the same row: its next token, drafted or not, is distributed as the target says. The count of a token of
    probability p is within 5 of its deviations sqrt(n p (1 - p)) of n p (one in a million falls outside)."""
    say("distribution")
    rng = np.random.default_rng(14)
    p, q = np.array([0.45, 0.05, 0.3, 0.15, 0.05]), np.array([0.1, 0.4, 0.3, 0.0, 0.2])
    B, n = 4096, 4                                                   # three drafts of what follows row 0
    off = (np.arange(B + 1) * n).astype(np.int32)
    parent = np.tile(np.array([-1, 0, 0, 0], np.int32), B)
    rows = np.tile(p.astype(np.float32), (B * n, 1))
    for drawn in (True, False):
        tokens = rng.choice(5, size=B * n, p=q).astype(np.int32)
        draft = R.DeviceDraft(t(off), torch.zeros(B * n, dtype=torch.int32, device="cuda"),
                              torch.zeros(B * n, dtype=torch.int64, device="cuda"), max_rows=n)
        v = R.DraftVerifier(B, 2, 5)
        v.run(draft, t(tokens), t(parent), t(rows), t(rng.random(B * n).astype(np.float32)), t(rng.random(B).astype(np.float32)),
              proposal=t(np.tile(q.astype(np.float32), (B * n, 1))) if drawn else None)
        path, nxt = v.path.cpu().numpy(), v.next.cpu().numpy()
        first = np.where(path[:, 1] >= 0, tokens[np.arange(B) * n + np.maximum(path[:, 1], 0)], nxt)
        assert 0.2 < (path[:, 1] >= 0).mean() < 0.999
        for x in range(5):
            assert abs((first == x).sum() - B * p[x]) <= 5 * np.sqrt(B * p[x] * (1 - p[x])), (drawn, x)


def test_another_stream_and_a_captured_run():
    say("graph")
    c = Case([5, 9, 1, 7], 3001, 2, True, seed=15)
    v, draft, args = R.DraftVerifier(4, 9, 3001), c.draft(), c.args()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        v.run(draft, *args, proposal=c.proposal)
    torch.cuda.synchronize()
    path, lens, nxt = c.expect()
    np.testing.assert_array_equal(v.path.cpu().numpy(), path)
    np.testing.assert_array_equal(v.next.cpu().numpy(), nxt)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        v.run(draft, *args, proposal=c.proposal)
    for i in range(3):
        c.u[:], c.v[:] = c.rng.random(c.rows), c.rng.random(4)
        args[3].copy_(t(c.u))
        args[4].copy_(t(c.v))
        v.path.fill_(-9)
        g.replay()
        torch.cuda.synchronize()
        path, lens, nxt = c.expect()
        np.testing.assert_array_equal(v.path.cpu().numpy(), path)
        np.testing.assert_array_equal(v.path_len.cpu().numpy(), lens)
        np.testing.assert_array_equal(v.next.cpu().numpy(), nxt)
