"""Counts past one launch's grid: 2^24 workgroups of 256 threads are one more than a launch dimension takes."""
import sys

import numpy as np
import pytest
import torch

import workloads as W

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402

MANY = (1 << 24) + 5


@pytest.mark.parametrize("interleaved", [True, False])
def test_rotary_rows(interleaved):
    """The rows of every launch equal those of a call on them alone; a negative position is left alone in each."""
    print("[case] many rows: rope", interleaved, file=sys.stderr, flush=True)
    r = R.Rope(16, rotary_dim=8 if interleaved else 6, interleaved=interleaved)
    x = torch.randn(1 << 20, 1, 16, device="cuda").to(torch.bfloat16).repeat(MANY // (1 << 20) + 1, 1, 1)[:MANY].contiguous()
    pos = torch.arange(MANY, dtype=torch.int32, device="cuda") * 3 % 100003
    left = torch.tensor([0, 77, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, MANY - 1], device="cuda")
    pos[left[1:-1]] = -1
    out = torch.full_like(x, 7.0)
    R.rope(r, x, pos, out=out)
    torch.cuda.synchronize()
    assert (out[left[1:-1]] == 7.0).all()
    part = torch.full((1000, 1, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    for at in (0, 5000, (1 << 23) - 500, MANY - 1500, MANY - 1000):
        rows = slice(at, at + 1000)
        part.fill_(7.0)
        R.rope(r, x[rows].clone(), pos[rows].clone(), out=part)
        assert torch.equal(out[rows], part), at
    assert int((out.view(-1, 16) == 7.0).all(dim=1).sum()) == len(left) - 2


def test_page_copies():
    """Nearly all pairs copy a page to itself, which is nothing; the others lie at the ends of what a launch takes."""
    print("[case] many rows: copies", file=sys.stderr, flush=True)
    cfg = W.LayerCfg(hidden=256, n_q=1, n_kv=1, head_dim=64, ffn=512)
    pool = torch.randn(40, 2, 1, 16 * 64, device="cuda").to(torch.bfloat16)
    block = R.DeviceBlock([cfg], [{}], [pool], 40)
    pairs = torch.zeros(MANY, 2, dtype=torch.int32, device="cuda")
    at = [0, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, MANY - 1]
    for i, k in enumerate(at):
        pairs[k] = torch.tensor([2 * i + 1, 2 * i + 2], dtype=torch.int32)
    want = pool.clone()
    for i in range(len(at)):
        want[2 * i + 2] = pool[2 * i + 1]
    R.kv_copy_pages(block, pairs)
    torch.cuda.synchronize()
    assert torch.equal(pool.view(torch.int16), want.view(torch.int16))
