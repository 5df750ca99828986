"""Rotary positions (ods_rope_rows) against the formula in 64 bits, element by element: layouts, parts of the head,
scalings, strides, far positions, in place and beside, skipped rows."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402


def say(*a):
    print("[case] rope", *a, file=sys.stderr, flush=True)


def make(rows, heads, extra, hd, seed, pos_hi):
    rng = np.random.default_rng(seed)
    full = torch.from_numpy(rng.standard_normal((rows, heads + extra, hd)).astype(np.float32)).to(torch.bfloat16).cuda()
    pos = rng.integers(0, pos_hi, rows).astype(np.int32)
    return full, pos


def expect(x, pos, r, f):
    xd = x.double().cpu().numpy()
    y = D.rotate(xd, pos, f, r.c.rotary_dim, r.c.interleaved, r.c.amplitude)
    return y, D.rotate_bound(xd, y, r.c.rotary_dim, r.c.interleaved, r.c.amplitude)


def check(got, y, bound):
    d = np.abs(got.double().cpu().numpy() - y)
    assert (d <= bound).all(), f"worst {np.nanmax(d - bound)} over the bound at {np.unravel_index(np.nanargmax(d - bound), d.shape)}"


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,rdim", [(64, 64), (128, 128), (128, 64), (128, 32), (256, 256), (96, 48), (64, 2), (64, 6),
                                     (72, 34), (8, 8), (8, 4), (128, 120), (256, 250)])
@pytest.mark.parametrize("rows,heads,extra", [(1, 1, 0), (3, 6, 2), (37, 40, 8), (700, 3, 1)])
def test_layouts_and_parts(rows, heads, extra, hd, rdim, interleaved):
    say(rows, heads, extra, hd, rdim, interleaved)
    full, pos = make(rows, heads, extra, hd, rows + hd + rdim, 5000)
    r = R.Rope(hd, rotary_dim=rdim, interleaved=interleaved, amplitude=1.25)
    x = full[:, :heads]
    y, bound = expect(x, pos, r, D.freqs(rdim, 1e4))
    before = full.clone()
    out = torch.full((rows, heads, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert R.rope(r, x, torch.from_numpy(pos).cuda(), out=out) is out
    check(out, y, bound)
    assert torch.equal(full, before)
    R.rope(r, x, torch.from_numpy(pos).cuda())                      # in place: the same bits, the other heads untouched
    assert torch.equal(full[:, :heads], out)
    assert torch.equal(full[:, heads:], before[:, heads:])


@pytest.mark.parametrize("scaling,kw", [("linear", {}), ("base", {}), ("rotations", {}), ("index", {}),
                                        ("index", dict(turns=(8, 2))), ("rotations", dict(turns=(9.5, 0.25)))])
def test_scalings_at_far_positions(scaling, kw):
    say(scaling, kw)
    full, pos = make(50, 5, 0, 128, 3, 2_000_000_000)
    pos[:4] = 0, 1, 2**31 - 1, 1_000_003
    r = R.Rope(128, theta=5e5, scaling=scaling, factor=16.0, orig_ctx=4096, **kw)
    hi, lo = kw.get("turns", (32, 1) if scaling == "index" else (4, 1))
    f = D.freqs(128, 5e5, scaling, 16.0, 4096, hi, lo)
    # the angle is below 2^31 and its double off by 2^-53 of it twice (product, reduction): under 2^-20 turns more
    y, bound = expect(full, pos, r, f)
    xd = full.double().cpu().numpy()
    bound[..., :64] += 2.0 ** -20 * (np.abs(xd[..., :64]) + np.abs(xd[..., 64:]))
    bound[..., 64:] += 2.0 ** -20 * (np.abs(xd[..., :64]) + np.abs(xd[..., 64:]))
    check(R.rope(r, full, torch.from_numpy(pos).cuda(), out=torch.empty_like(full)), y, bound)


def test_negative_positions_are_left_alone():
    say("skipped rows")
    for heads, extra, rows in ((6, 2, 9), (2, 0, 300)):
        full, pos = make(rows, heads, extra, 64, 11, 900)
        pos[::2] = -1 - np.arange(len(pos[::2]))
        r = R.Rope(64)
        y, bound = expect(full[:, :heads], np.maximum(pos, 0), r, D.freqs(64, 1e4))
        out = torch.full((rows, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        R.rope(r, full[:, :heads], torch.from_numpy(pos).cuda(), out=out)
        assert (out[0::2] == 7.0).all()
        check(out[1::2], y[1::2], bound[1::2])


def test_columns_of_the_same_rows_and_odd_strides():
    say("strides")
    r, rows = R.Rope(64, rotary_dim=32, interleaved=True), 21
    buf, pos = make(rows, 9, 0, 64, 5, 4000)
    wide = torch.zeros(rows, 9 * 64 + 24, dtype=torch.bfloat16, device="cuda")   # a stride of 600 values
    wide[:, :576] = buf.reshape(rows, -1)
    view = lambda c0, n: wide[:, c0:c0 + n * 64].unflatten(1, (n, 64))  # noqa: E731
    y, bound = expect(view(0, 3), pos, r, D.freqs(32, 1e4))
    keep = wide.clone()
    R.rope(r, view(0, 3), torch.from_numpy(pos).cuda(), out=view(5 * 64, 3))     # beside each other in one buffer
    check(view(5 * 64, 3), y, bound)
    assert torch.equal(wide[:, :320], keep[:, :320]) and torch.equal(wide[:, 512:], keep[:, 512:])
    y, bound = expect(view(8, 3), pos, r, D.freqs(32, 1e4))                      # rows that start 16 bytes in
    check(R.rope(r, view(8, 3), torch.from_numpy(pos).cuda(), out=torch.empty(rows, 3, 64, dtype=torch.bfloat16,
                                                                              device="cuda")), y, bound)


def test_infinities_and_nan_stay_in_their_pairs():
    say("non-finite")
    r = R.Rope(64)
    x = torch.ones(2, 3, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 1, 5] = float("nan")
    x[1, 2, 40] = float("inf")
    out = R.rope(r, x, torch.tensor([3, 9], dtype=torch.int32, device="cuda"), out=torch.empty_like(x))
    bad = ~torch.isfinite(out)
    assert bad.nonzero().tolist() == [[0, 1, 5], [0, 1, 37], [1, 2, 8], [1, 2, 40]]


def test_empty_calls():
    r = R.Rope(64)
    x = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    R.rope(r, x, torch.empty(0, dtype=torch.int32, device="cuda"))
    R.rope(r, torch.empty(4, 0, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"))


def test_another_stream():
    say("stream")
    full, pos = make(64, 8, 0, 128, 2, 100)
    r, p = R.Rope(128), torch.from_numpy(pos).cuda()
    want = R.rope(r, full, p, out=torch.empty_like(full))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = R.rope(r, full, p, out=torch.empty_like(full))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
