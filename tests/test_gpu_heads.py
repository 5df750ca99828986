"""Heads normalised and turned in one pass (ods_head_rows, and the rope operator of drafted rows with a norm) against the
formula in 64 bits, element by element: layouts, parts, axes, strides, skipped rows, in place, captured."""
import sys

import numpy as np
import pytest
import torch

import draft_ref as D
import serve_ref as S
import workloads as W

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2609_14237_amd import runtime as R  # noqa: E402


def say(*a):
    print("[case] heads", *a, file=sys.stderr, flush=True)


def bf(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).cuda()


def make(rows, heads, extra, hd, seed, pos_hi, axes=1):
    rng = np.random.default_rng(seed)
    full = bf(rng.standard_normal((rows, heads + extra, hd)) * np.exp(rng.standard_normal((rows, heads + extra, 1))))
    pos = rng.integers(0, pos_hi, (rows, axes)).astype(np.int32)
    return full, pos, bf(1 + 0.3 * rng.standard_normal(hd)), bf(1 + 0.3 * rng.standard_normal(hd))


def f64(t):
    return t.double().cpu().numpy()


def check(got, y, bound):
    d = np.abs(f64(got) - y)
    assert (d <= bound).all(), f"worst {np.nanmax(d - bound)} over the bound at {np.unravel_index(np.nanargmax(d - bound), d.shape)}"


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,rdim", [(64, 64), (128, 128), (128, 64), (128, 32), (256, 256), (96, 48), (64, 2), (64, 6),
                                     (80, 80), (80, 40), (72, 34), (8, 8), (8, 4), (128, 120), (256, 250)])
@pytest.mark.parametrize("rows,n_q,n_k,extra", [(1, 1, 0, 0), (3, 4, 2, 2), (37, 32, 8, 8), (700, 2, 1, 1), (65, 1, 0, 0)])
def test_layouts_and_parts(rows, n_q, n_k, extra, hd, rdim, interleaved):
    say(rows, n_q, n_k, extra, hd, rdim, interleaved)
    heads = n_q + n_k
    full, pos, gq, gk = make(rows, heads, extra, hd, rows + hd + rdim, 5000)
    r = R.Rope(hd, rotary_dim=rdim, interleaved=interleaved, amplitude=1.25)
    norm = R.HeadNorm(gq, gk, n_q=n_q, eps=1e-5)
    x, p = full[:, :heads], torch.from_numpy(pos[:, 0].copy()).cuda()
    y, bound = S.heads(f64(x), pos, [0] * (rdim // 2), D.freqs(rdim, 1e4), rdim, interleaved, f64(gq), f64(gk), n_q, 1e-5, 1.25)
    before = full.clone()
    out = torch.full((rows, heads, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert R.rope(r, x, p, out=out, norm=norm) is out
    check(out, y, bound)
    assert torch.equal(full, before)
    R.rope(r, x, p, norm=norm)                      # in place: the same bits, the other heads untouched
    assert torch.equal(full[:, :heads], out)
    assert torch.equal(full[:, heads:], before[:, heads:])


@pytest.mark.parametrize("with_norm", [False, True])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("order", ["blocks", "cyclic"])
@pytest.mark.parametrize("hd,rdim,sections", [(128, 128, (16, 24, 24)), (128, 64, (8, 12, 12)), (64, 64, (16, 16)), (64, 64, (32,)),
                                              (80, 36, (0, 7, 11)), (64, 32, (1, 1, 2, 2, 3, 3, 4, 0))])
def test_axes(hd, rdim, sections, order, own, with_norm):
    say("axes", hd, rdim, sections, order, own, with_norm)
    rows, n_q, n_k = 45, 5, 2
    full, pos, gq, gk = make(rows, 7, 1, hd, hd + rdim, 3000, len(sections))
    axis, f = S.section_freqs(sections, order, 5e5, rdim, own)
    r = R.Rope(hd, theta=5e5, rotary_dim=rdim, sections=sections, order=order, own_freqs=own)
    norm = R.HeadNorm(gq, gk, n_q=n_q) if with_norm else None
    x = full[:, :7]
    y, bound = S.heads(f64(x), pos, axis, f, rdim, False, *((f64(gq), f64(gk), n_q, 1e-6) if with_norm else ()))
    check(R.rope(r, x, torch.from_numpy(pos).cuda(), out=torch.empty(rows, 7, hd, dtype=torch.bfloat16, device="cuda"), norm=norm),
          y, bound)


def test_rows_with_a_negative_position_are_left_alone():
    say("skipped rows")
    for sections, heads in (((10, 22), 3), (None, 40)):
        axes = len(sections or (0,))
        full, pos, gq, _ = make(301, heads, 0, 64, 3, 900, axes)
        pos[::3, -1] = -1
        r = R.Rope(64, sections=sections)
        axis, f = S.section_freqs(sections or (32,), "blocks", 1e4, 64, False)
        y, bound = S.heads(f64(full), np.maximum(pos, 0), axis, f, 64, False, f64(gq), None, heads, 1e-6)
        out = torch.full((301, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        R.rope(r, full, torch.from_numpy(pos if sections else pos[:, 0].copy()).cuda(), out=out, norm=R.HeadNorm(gq))
        live = (pos >= 0).all(1)
        assert (out[torch.from_numpy(~live).cuda()] == 7.0).all()
        check(out[torch.from_numpy(live).cuda()], y[live], bound[live])


def test_far_positions_strides_and_one_kind_of_head():
    say("far, strides")
    full, pos, gq, gk = make(33, 9, 0, 64, 8, 2_000_000_000)
    wide = torch.zeros(33, 9 * 64 + 24, dtype=torch.bfloat16, device="cuda")   # a stride of 600 values
    wide[:, 8:584] = full.reshape(33, -1)
    x = wide[:, 8:584].unflatten(1, (9, 64))
    p = torch.from_numpy(pos[:, 0].copy()).cuda()
    r = R.Rope(64, theta=5e5)
    for norm, n_q, gains in ((R.HeadNorm(gq), 9, (f64(gq), None)), (R.HeadNorm(gq, gk, n_q=0), 0, (f64(gq), f64(gk)))):
        y, bound = S.heads(f64(x), pos, [0] * 32, D.freqs(64, 5e5), 64, False, *gains, n_q, 1e-6)
        v = np.abs(y).max(-1, keepdims=True)
        bound = bound + 2.0 ** -20 * 2 * v  # the angle's double is off by 2^-53 of 2^31 twice
        check(R.rope(r, x, p, out=torch.empty(33, 9, 64, dtype=torch.bfloat16, device="cuda"), norm=norm), y, bound)


def test_zero_heads_and_what_is_not_finite():
    """A head of zeros stays zero with eps; infinities and NaN stay in their head."""
    say("non-finite")
    x = torch.ones(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 1], x[1, 2, 5], x[2, 0, 40] = 0.0, float("nan"), float("inf")
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = R.rope(R.Rope(64), x, torch.tensor([3, 9, 1], dtype=torch.int32, device="cuda"), out=torch.empty_like(x), norm=R.HeadNorm(g))
    assert (out[0, 1] == 0).all()
    bad = ~torch.isfinite(out)
    assert bad.any(-1).nonzero().tolist() == [[1, 2], [2, 0]]


def test_empty_calls_refusals_and_another_stream():
    say("empty, stream")
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    r, norm, z = R.Rope(64), R.HeadNorm(g), lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    R.rope(r, torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), z(0), norm=norm)
    R.rope(r, torch.empty(4, 0, 64, dtype=torch.bfloat16, device="cuda"), z(4), norm=norm)
    x = torch.randn(9, 4, 64, device="cuda").to(torch.bfloat16)
    with pytest.raises(ValueError):
        R.rope(r, x, z(9), norm=R.HeadNorm(g, n_q=3))
    with pytest.raises(ValueError, match="current device"):
        R.rope(r, x, z(9), norm=R.HeadNorm(g.cpu()))
    with pytest.raises(ValueError):
        R.rope(R.Rope(64, sections=(16, 16)), x, z(9))
    want = R.rope(r, x, z(9) + 5, out=torch.empty_like(x), norm=norm)
    p, got = z(9) + 5, torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        R.rope(r, x, p, out=got, norm=norm)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_more_heads_than_a_block_divides():
    """Rows of 2^13 heads and more, several rows, odd counts of them around the blocks'."""
    say("wide rows")
    for heads, rows in ((8191, 3), (8192, 3), (9001, 2), (5, 2049), (3, 4100), (40, 2050)):
        full, pos, gq, gk = make(rows, heads, 0, 8, heads, 3000)
        y, bound = S.heads(f64(full), pos, [0] * 4, D.freqs(8, 1e4), 8, False, f64(gq), f64(gk), heads // 3, 1e-6)
        check(R.rope(R.Rope(8), full, torch.from_numpy(pos[:, 0].copy()).cuda(), out=torch.empty_like(full),
                     norm=R.HeadNorm(gq, gk, n_q=heads // 3)), y, bound)


def test_captured_and_replayed():
    say("graph")
    full, pos, gq, gk = make(20, 6, 0, 128, 4, 4000)
    r, norm, p = R.Rope(128), R.HeadNorm(gq, gk, n_q=4), torch.from_numpy(pos[:, 0].copy()).cuda()
    out = torch.empty_like(full)
    R.rope(r, full, p, out=out, norm=norm)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.rope(r, full, p, out=out, norm=norm)
    for i in range(3):
        p.add_(17)
        full.mul_(-1)
        want = R.rope(r, full, p, out=torch.empty_like(full), norm=norm)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


@pytest.mark.parametrize("hd,rdim,interleaved", [(64, None, False), (64, 24, True), (64, 20, False), (128, 64, False)])
def test_rope_operator_of_drafted_rows(hd, rdim, interleaved):
    """run_draft's rope (and kv_append) normalises q and k, leaves v, and skips sequences that are left alone."""
    say("drafted", hd, rdim, interleaved)
    n_q, n_kv = 4, 2
    ctx, counts = np.array([0, 5, -1, 300], np.int32), [3, 1, 2, 9]
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rng = np.random.default_rng(hd)
    rows = int(off[-1]) + 2                                       # two rows of padding
    qkv = bf(rng.standard_normal((rows, n_q + 2 * n_kv, hd)) * 3)
    gq, gk = bf(1 + 0.3 * rng.standard_normal(hd)), bf(1 + 0.3 * rng.standard_normal(hd))
    depth = np.concatenate([np.arange(c) for c in counts] + [[0, 0]]).astype(np.int32)
    pages = 20
    table = rng.permutation(4 * pages).reshape(4, pages).astype(np.int32)
    cfg = W.LayerCfg(hidden=256, n_q=n_q, n_kv=n_kv, head_dim=hd, ffn=512)
    pool = torch.zeros(4 * pages, 2, n_kv, 16 * hd, dtype=torch.bfloat16, device="cuda")
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    block = R.DeviceBlock([cfg], [{}], [pool], 4 * pages)
    batch = R.DeviceBatch(t(ctx), t(table))
    rope = None if rdim is None else [R.Rope(hd, rotary_dim=rdim, interleaved=interleaved)]
    draft = R.DeviceDraft(t(off), t(depth), torch.ones(rows, dtype=torch.int64, device="cuda"), max_rows=9, rope=rope,
                          norm=[R.HeadNorm(gq, gk, eps=1e-6)])
    state = R.DeviceState(block, batch, draft=draft)
    v = state.view("qkv", rows, n_q + 2 * n_kv, hd)
    v.copy_(qkv)
    R.run_draft(block, 2, 4, batch, draft, state)
    torch.cuda.synchronize()
    r = rdim or hd
    pos = np.concatenate([[c + d for d in range(n)] for c, n in zip(ctx, counts)] + [[0, 0]])[:, None]
    y, bound = S.heads(f64(qkv[:, :n_q + n_kv]), np.maximum(pos, 0), [0] * (r // 2), D.freqs(r, 1e4), r, interleaved, f64(gq), f64(gk),
                       n_q, 1e-6)
    live = np.r_[0:4, 6:15]
    check(v[live][:, :n_q + n_kv], y[live], bound[live])
    assert torch.equal(v[:, n_q + n_kv:], qkv[:, n_q + n_kv:])
    rest = [4, 5, 15, 16]
    assert torch.equal(v[rest], qkv[rest])
    hp = f64(pool)
    for b in (0, 1, 3):
        for j in range(counts[b]):
            k, val = D.slot(hp, table[b], int(ctx[b]) + j, 0, n_kv, hd)
            row = f64(v[int(off[b]) + j])
            np.testing.assert_array_equal(k, row[n_q:n_q + n_kv])
            np.testing.assert_array_equal(val, row[n_q + n_kv:])
