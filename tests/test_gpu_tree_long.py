"""Drafted rows' attention where a workgroup's range passes several tasks and more than one window of page ids (32 tiles), at
the widths whose kernels have no registers to spare, against the definition in 64 bits, computed on the GPU; and what is not
finite in any block of dims there."""
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


def say(*a):
    print("[case] long", *a, file=sys.stderr, flush=True)


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("B,n,g,hd,window,lo,hi", [
    (300, 24, 8, 128, 0, 500, 3000),     # 192 columns: eight waves of 32
    (300, 64, 4, 128, 0, 500, 3000),     # 256
    (600, 16, 8, 128, 1500, 1000, 6000),  # 128 behind a window: four waves of 32
    (300, 24, 8, 64, 0, 500, 3000),
    (600, 16, 8, 64, 1500, 1000, 6000),
    (700, 16, 8, 128, 0, 100, 2000),     # 128: eight waves of 16
    (700, 6, 8, 128, 0, 100, 2000),      # 48: four waves
])
def test_ranges_of_several_tasks(B, n, g, hd, window, lo, hi):
    say(B, n, g, hd, window)
    rng = np.random.default_rng(B + n + hd)
    ctx = rng.integers(lo, hi, B)
    first = np.maximum(ctx - window + 1, 0) // PAGE if window else np.zeros(B, np.int64)
    end = -(-(ctx + n) // PAGE)
    P = int((end - first).sum())
    ids, at = rng.permutation(P).astype(np.int32), 0
    table = np.full((B, int(end.max())), -1, np.int32)
    for b in range(B):
        k = int(end[b] - first[b])
        table[b, first[b]:end[b]] = ids[at:at + k]
        at += k
    gen = torch.Generator(device="cuda").manual_seed(hd + n)
    pool = torch.randn((P, 2, 1, PAGE * hd), generator=gen, device="cuda").to(torch.bfloat16)
    qkv = torch.randn((B * n, (g + 2) * hd), generator=gen, device="cuda").to(torch.bfloat16)
    block = R.DeviceBlock([W.LayerCfg(hidden=256, n_q=g, n_kv=1, head_dim=hd, ffn=512, window=window)], [{}], [pool], P)
    batch = R.DeviceBatch(cuda(ctx.astype(np.int32)), cuda(table))
    words = -(-n // 64)
    mask = D.mask_words([list(range(j + 1)) for j in range(n)], n)   # a chain: rows see those before them
    draft = R.DeviceDraft(cuda(np.arange(B + 1, dtype=np.int32) * n), cuda(np.tile(np.arange(n, dtype=np.int32), B)),
                          cuda(np.tile(mask, (B, 1)).reshape(B * n, words)), max_rows=n)
    state = R.DeviceState(block, batch, fill=float("nan"), draft=draft)
    state.view("qkv", *qkv.shape).copy_(qkv)
    R.run_draft(block, 4, 5, batch, draft, state)
    torch.cuda.synchronize()
    got = state.view("o", B * n, g * hd).double().cpu().numpy().reshape(B, n, g, hd)
    row = torch.arange(n, device="cuda")[:, None, None]
    for b in range(B):
        c, last, t0 = int(ctx[b]), int(ctx[b]) + n, int(first[b]) * PAGE
        pages = pool[torch.from_numpy(table[b, first[b]:end[b]].astype(np.int64)).cuda()].double()
        k = pages[:, 0, 0].reshape(-1, hd)[:last - t0]
        v = pages[:, 1, 0].view(-1, hd, PAGE).transpose(1, 2).reshape(-1, hd)[:last - t0]
        s = (qkv[b * n:(b + 1) * n, :g * hd].double().reshape(n * g, hd) @ k.T / hd ** 0.5).view(n, g, last - t0)
        t = torch.arange(t0, last, device="cuda")
        hidden = t > c + row
        if window:
            hidden = hidden | (t < c + row - window + 1)
        p = torch.softmax(s.masked_fill(hidden, -float("inf")), dim=2).view(n * g, last - t0)
        o, mag = ((p @ x).cpu().numpy().reshape(n, g, hd) for x in (v, v.abs()))
        off = np.abs(got[b] - o) - D.tree_bound(o, mag)
        assert (off <= 0).all(), f"sequence {b}: off by {off.max()} more than the bound"


@pytest.mark.parametrize("hd,rows", [(128, 40), (128, 20), (128, 10), (128, 3), (64, 40)])
def test_what_is_not_finite_in_some_dims(hd, rows):
    """Infinities and NaN in a few dims of drafted tokens, each block of sixteen dims in turn: rows that see them get them in
    those dims, all else is what it was."""
    say("dims", hd, rows)
    c = Case([70, 90, 33], [rows, 2, rows - 1], n_q=8, n_kv=2, hd=hd, seed=hd + rows, max_rows=rows)
    c.device()
    plain = c.attend()
    c.check(plain)
    bad = [float("nan"), float("inf"), -float("inf")]
    for b in (0, 2):
        for i, d in enumerate(range(5, hd, 16)):
            t = int(c.ctx[b]) + i % (rows - 1)
            for h in range(2):
                c.pool[c.table[b, t // PAGE]].view(2, 2, PAGE * hd)[1].view(2, hd, PAGE)[h, d + h, t % PAGE] = bad[(i + h + b) % 3]
    c.device()
    got = c.attend()
    c.check(got)
    seen = ~torch.isfinite(got)
    assert seen.any() and torch.equal(got[~seen], plain[~seen])
    for d in range(hd):
        if d % 16 not in (5, 6):
            assert not seen.view(c.R, 8, hd)[..., d].any()
