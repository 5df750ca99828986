"""Rows of several axes in a drafted step: positions that are not the cache's (an image in the prompt) are turned by R.rope on
the state's qkv between the operators, in place of the step's own rope."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D
import serve_ref as S

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402
from test_gpu_tree import Case  # noqa: E402

PAGE = 16


@pytest.mark.parametrize("n_q,n_kv,hd,rdim,sections,order", [(8, 2, 64, 64, (8, 12, 12), "cyclic"), (4, 1, 128, 64, (16, 8, 8), "blocks"),
                                                             (6, 3, 128, 100, (10, 20, 20), "cyclic")])
def test_step_with_positions_of_its_own(n_q, n_kv, hd, rdim, sections, order):
    print("[case] axes", n_q, n_kv, hd, rdim, file=sys.stderr, flush=True)
    c = Case([90, 33, 200], [5, 1, 12], n_q, n_kv, hd, seed=hd + rdim).device()
    rng = np.random.default_rng(rdim)
    gains = [torch.from_numpy(1 + 0.2 * rng.standard_normal(hd)).to(torch.bfloat16).cuda() for _ in range(2)]
    r, norm = R.Rope(hd, theta=1e6, rotary_dim=rdim, sections=sections, order=order), R.HeadNorm(*gains, n_q=n_q)
    # an image of 40 tokens took 40 slots of the cache and 8 positions; its rows and columns are the other axes
    text = np.repeat(c.ctx, c.n) + c.depth - 32
    pos = np.stack([text, text + rng.integers(0, 7, c.R), text + rng.integers(0, 5, c.R)], 1).astype(np.int32)
    heads = n_q + n_kv
    qkv = c.state.view("qkv", c.R, heads + n_kv, hd)
    x = qkv[:, :heads].double().cpu().numpy()
    v = qkv[:, heads:].clone()
    R.rope(r, qkv[:, :heads], torch.from_numpy(pos).cuda(), norm=norm)
    R.run_draft(c.block, 3, 5, c.batch, c.draft, c.state)   # append, attention
    torch.cuda.synchronize()
    axis, f = S.section_freqs(sections, order, 1e6, rdim, False)
    y, bound = S.heads(x, pos, axis, f, rdim, False, *(g.double().cpu().numpy() for g in gains), n_q=n_q, eps=1e-6)
    assert (np.abs(qkv[:, :heads].double().cpu().numpy() - y) <= bound).all() and torch.equal(qkv[:, heads:], v)
    for b in range(3):                                      # what was appended is what was turned
        for j in range(int(c.n[b])):
            t, row = int(c.ctx[b]) + j, int(c.off[b]) + j
            k = c.dpool.view(c.P, 2, n_kv, PAGE, hd)[int(c.table[b, t // PAGE]), 0, :, t % PAGE]
            assert torch.equal(k, qkv[row, n_q:heads])
    c.check(c.o().clone(), pool=c.dpool.cpu(), qkv=qkv.reshape(c.R, -1).cpu())


def test_text_rows_are_the_step_s_own():
    """With every axis at the row's position both ways give the same bits."""
    c, gains = Case([70, 31], [6, 3], 8, 2, 64, seed=4), [torch.ones(64, dtype=torch.bfloat16, device="cuda")] * 2
    r = R.Rope(64, sections=(10, 11, 11), order="cyclic")
    c.device([r])
    c.draft = R.DeviceDraft(c.draft.row_off, c.draft.depth, c.draft.mask, max_rows=c.max_rows, rope=[r], norm=[R.HeadNorm(*gains)])
    R.run_draft(c.block, 2, 5, c.batch, c.draft, c.state)
    whole = (c.state.view("qkv", *c.qkv.shape).clone(), c.o().clone(), c.dpool.clone())
    c.device([r])
    qkv = c.state.view("qkv", c.R, 12, 64)
    text = np.repeat(c.ctx, c.n) + c.depth
    R.rope(r, qkv[:, :10], torch.from_numpy(np.repeat(text[:, None], 3, 1).astype(np.int32)).cuda(), norm=R.HeadNorm(*gains, n_q=8))
    R.run_draft(c.block, 3, 5, c.batch, c.draft, c.state)
    torch.cuda.synchronize()
    assert torch.equal(c.state.view("qkv", *c.qkv.shape), whole[0]) and torch.equal(c.o(), whole[1])
    np.testing.assert_array_equal(D.bits(c.dpool), D.bits(whole[2]))
