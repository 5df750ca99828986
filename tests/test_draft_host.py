"""Host-side checks, without a GPU, of rotary positions, drafted rows and the page bookkeeping: frequency tables
against their formulas, every refusal (all return before anything is enqueued), pages against a plain model, and the
HIP-free sources under the CPU sanitizers."""
import ctypes as C
import os
import shutil
import subprocess
from dataclasses import replace

import numpy as np
import pytest

import draft_ref as D
import workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = os.environ.get("CXX", "g++")

B = pytest.importorskip("paper_2609_14237_amd.binding")
from paper_2609_14237_amd import runtime as R  # noqa: E402

FAKE = 0x10000  # aligned, never dereferenced: every call below fails its checks or has nothing to do


class _Fake:
    def data_ptr(self):
        return FAKE


CFG = W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512)


def rope_struct(**kw):
    f = dict(head_dim=128, rotary_dim=128, interleaved=0, scaling=0, theta=1e4, factor=4.0, orig_ctx=8192.0,
             turns_hi=4.0, turns_lo=1.0, amplitude=1.0, freqs=FAKE)
    f.update(kw)
    return B.ods_rope(*[f[n] for n, _ in B.ods_rope._fields_])


@pytest.mark.parametrize("scaling,hi,lo", [("plain", 4, 1), ("linear", 4, 1), ("base", 4, 1), ("rotations", 4, 1),
                                           ("rotations", 9.5, 0.25), ("index", 32, 1), ("index", 8, 2)])
@pytest.mark.parametrize("hd,rdim,theta,factor,orig", [(128, 128, 1e4, 8.0, 8192), (64, 24, 5e5, 2.0, 4096),
                                                       (256, 2, 1e6, 32.0, 2048), (96, 94, 1e4, 1.0, 100)])
def test_rope_freqs_follow_their_formulas(hd, rdim, theta, factor, orig, scaling, hi, lo):
    r = rope_struct(head_dim=hd, rotary_dim=rdim, scaling=R.Rope.SCALINGS[scaling], theta=theta, factor=factor,
                    orig_ctx=orig, turns_hi=hi, turns_lo=lo, freqs=None)
    got = np.zeros(rdim // 2)
    assert B.ods_rope_freqs(r, got) == B.ODS_OK
    np.testing.assert_allclose(got, D.freqs(rdim, theta, scaling, factor, orig, hi, lo), rtol=1e-13)


@pytest.mark.parametrize("bad,status", [
    (dict(head_dim=0), B.ODS_EINVAL), (dict(head_dim=100, rotary_dim=64), B.ODS_EUNSUPPORTED),
    (dict(head_dim=264), B.ODS_EUNSUPPORTED), (dict(rotary_dim=0), B.ODS_EINVAL), (dict(rotary_dim=3), B.ODS_EINVAL),
    (dict(rotary_dim=130), B.ODS_EINVAL), (dict(interleaved=2), B.ODS_EINVAL), (dict(scaling=5), B.ODS_EINVAL),
    (dict(scaling=-1), B.ODS_EINVAL), (dict(theta=0.0), B.ODS_EINVAL), (dict(theta=float("nan")), B.ODS_EINVAL),
    (dict(theta=float("inf")), B.ODS_EINVAL), (dict(amplitude=float("inf")), B.ODS_EINVAL),
    (dict(scaling=1, factor=0.0), B.ODS_EINVAL), (dict(scaling=3, orig_ctx=-1.0), B.ODS_EINVAL),
    (dict(scaling=3, turns_lo=4.0), B.ODS_EINVAL), (dict(scaling=4, turns_lo=0.0), B.ODS_EINVAL),
    (dict(scaling=4, theta=1.0), B.ODS_EINVAL)])
def test_rope_fields_are_refused(bad, status):
    r = rope_struct(**bad)
    assert B.ods_rope_freqs(r, np.zeros(256)) == status
    assert B.ods_rope_rows(r, FAKE, 256, FAKE, 256, 4, 2, FAKE, None) == status


def test_rope_rows_arguments():
    r, far = rope_struct(), FAKE + (1 << 20)
    call = lambda **k: B.ods_rope_rows(k.get("r", r), k.get("x", FAKE), k.get("xs", 512), k.get("y", far),  # noqa: E731
                                       k.get("ys", 256), k.get("rows", 4), k.get("heads", 2), k.get("pos", FAKE), None)
    assert B.lib.ods_rope_rows(None, FAKE, 512, far, 512, 4, 2, FAKE, None) == B.ODS_EINVAL
    assert B.lib.ods_rope_freqs(C.byref(r), None) == B.ODS_EINVAL
    for bad in (dict(x=None), dict(y=None), dict(pos=None), dict(pos=FAKE + 2), dict(x=FAKE + 8), dict(y=far + 2),
                dict(rows=-1), dict(heads=-1), dict(xs=248), dict(ys=255), dict(ys=260), dict(xs=-512),
                dict(r=rope_struct(freqs=None)), dict(r=rope_struct(freqs=FAKE + 8)), dict(xs=1 << 62)):
        assert call(**bad) == B.ODS_EINVAL, bad
    # overlaps: other columns of the same rows are fine (they reach the launch, so rows = 0 here is all that can be run)
    assert call(rows=0, x=None) == B.ODS_OK and call(heads=0, y=None) == B.ODS_OK
    for y, ys in ((FAKE + 16, 512), (FAKE + 256 * 2 - 16, 512), (FAKE, 256), (FAKE + 512 * 2 * 3, 256),
                  (FAKE + 512 * 2 - 256 * 2 + 16, 512)):
        assert call(y=y, ys=ys) == B.ODS_EINVAL, (y, ys)
        assert "overlap" in B.ods_last_error()


def fake_draft(rope=None, **kw):
    f = dict(rows=8, max_rows=4, row_off=FAKE, depth=FAKE, mask=FAKE)
    f.update(kw)
    return B.ods_draft(f["rows"], f["max_rows"], f["row_off"], f["depth"], f["mask"],
                       None if rope is None else C.cast(rope, C.POINTER(B.ods_rope)))


def fake_block(cfgs):
    ws = [{k: _Fake() for k in ("g_attn", "w_qkv", "w_o", "g_ffn", "w_gate_up", "w_down", "w_router")} for _ in cfgs]
    return R.DeviceBlock(cfgs, ws, [_Fake()] * len(cfgs), 100)


def fake_batch(**kw):
    f = dict(batch=2, max_pages=8, ctx_lens=FAKE, page_table=FAKE, split_pages=0, ring_pages=0, ring_table=None)
    f.update(kw)
    return B.ods_batch(*[f[n] for n, _ in B.ods_batch._fields_])


def fake_state(**kw):
    s = B.ods_state()
    for name in B.BUFFERS:
        setattr(s, name, FAKE)
    s.ws, s.ws_bytes = FAKE, 1 << 40
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_run_draft_refusals():
    blk = fake_block([CFG, replace(CFG, window=40)])
    run = lambda a, b, batch=None, draft=None, st=None: B.ods_run_draft(  # noqa: E731
        blk.c, a, b, batch or fake_batch(), draft or fake_draft(), st or fake_state(), None)
    for a, b in ((-1, 3), (3, 3), (4, 2), (0, 21)):
        assert run(a, b) == B.ODS_ERANGE
    for d in (dict(rows=-1), dict(max_rows=0), dict(max_rows=257), dict(max_rows=-3)):
        assert run(2, 5, draft=fake_draft(**d)) == B.ODS_EINVAL, d
    for name in ("row_off", "depth", "mask"):
        assert run(2, 5, draft=fake_draft(**{name: None})) == B.ODS_EINVAL
        assert name in B.ods_last_error()
        assert run(2, 5, draft=fake_draft(**{name: FAKE + 8})) == B.ODS_EINVAL
    for name in ("ctx_lens", "page_table"):
        assert run(2, 5, batch=fake_batch(**{name: None})) == B.ODS_EINVAL
    for name in ("qkv", "o"):
        assert run(4, 5, st=fake_state(**{name: None})) == B.ODS_EINVAL
        assert run(4, 5, st=fake_state(**{name: FAKE + 2})) == B.ODS_EINVAL
    assert run(2, 5, batch=fake_batch(batch=-1)) == B.ODS_EINVAL
    assert run(2, 5, batch=fake_batch(max_pages=0)) == B.ODS_EINVAL
    assert run(2, 5, batch=fake_batch(max_pages=1 << 28)) == B.ODS_ERANGE
    assert run(2, 5, batch=fake_batch(batch=4097)) == B.ODS_EUNSUPPORTED
    assert run(4, 5, draft=fake_draft(rows=1 << 30)) == B.ODS_EUNSUPPORTED
    # the whole range is checked before any of it runs: a bad later operator refuses the earlier ones
    assert run(0, 10, st=fake_state(act=None)) == B.ODS_EINVAL
    assert run(0, 5, st=fake_state(ws=None)) == B.ODS_EINVAL
    assert run(0, 5, st=fake_state(ws_bytes=16)) == B.ODS_ENOMEM
    # a ring holds the window and the drafted rows: ceil((40 + 4) / 16) + 1 = 4 pages
    assert run(14, 15, batch=fake_batch(ring_pages=3, ring_table=FAKE)) == B.ODS_EINVAL
    assert "ring_pages" in B.ods_last_error()
    assert run(14, 15, batch=fake_batch(ring_pages=4, ring_table=None)) == B.ODS_EINVAL
    ropes = (B.ods_rope * 2)(rope_struct(head_dim=64, rotary_dim=64), rope_struct())
    assert run(12, 14, draft=fake_draft(rope=ropes)) == B.ODS_EINVAL and "head_dim" in B.ods_last_error()
    ropes[1] = rope_struct(head_dim=64, rotary_dim=64, freqs=None)
    assert run(12, 14, draft=fake_draft(rope=ropes)) == B.ODS_EINVAL
    # nothing to do
    assert run(0, 20, batch=fake_batch(batch=0, ctx_lens=None)) == B.ODS_OK
    assert run(0, 20, draft=fake_draft(rows=0, row_off=None)) == B.ODS_OK
    st, h = B.ods_draft_graph(blk.c, 3, 99, fake_batch(), fake_draft(), fake_state())
    assert st != B.ODS_OK and h is None
    assert B.lib.ods_draft_graph(C.byref(blk.c), 0, 1, C.byref(fake_batch()), C.byref(fake_draft()),
                                 C.byref(fake_state()), None) == B.ODS_EINVAL
    assert B.ods_draft_workspace_bytes(blk.c, fake_batch(), fake_draft()) > 0
    assert B.ods_draft_workspace_bytes(blk.c, fake_batch(), fake_draft(max_rows=300)) == 0


def test_python_side_refusals():
    import torch
    i32, bf = torch.int32, torch.bfloat16
    blk, z = fake_block([CFG]), lambda *s, dt=i32: torch.zeros(*s, dtype=dt)
    with pytest.raises(ValueError):
        R.DeviceDraft(z(3), z(8), z(8, 2, dt=torch.int64), max_rows=4)
    with pytest.raises(ValueError):
        R.DeviceDraft(z(3), z(8), z(8), max_rows=4)
    d = R.DeviceDraft(z(3), z(8), z(8, dt=torch.int64), max_rows=64)
    batch = R.DeviceBatch(z(3), z(3, 4))
    with pytest.raises(ValueError):
        R.run_draft(blk, 4, 5, batch, d, R.ods_state())
    with pytest.raises(ValueError):
        R.kv_accept(blk, R.DeviceBatch(z(2), z(2, 4)), d, z(3, 4), z(2))
    with pytest.raises(ValueError):
        R.kv_copy_pages(blk, z(4, 2, dt=torch.int64))
    with pytest.raises(ValueError):
        R.Rope(64, scaling="other", device="cpu")
    with pytest.raises(B.OdsError):
        R.Rope(64, rotary_dim=65, device="cpu")
    r = R.Rope(64, device="cpu")
    for x in (z(4, 2, 64, dt=torch.float32), z(4, 128, dt=bf), z(4, 64, 2, dt=bf).transpose(1, 2)):
        with pytest.raises(ValueError):
            R.rope(r, x, z(4))
    with pytest.raises(ValueError):
        R.rope(r, z(4, 2, 64, dt=bf), z(5))
    with pytest.raises(B.OdsError):  # rows of stride 0
        R.rope(r, z(1, 2, 64, dt=bf).expand(4, 2, 64), z(4), stream=0)


def test_page_operator_refusals():
    blk = fake_block([CFG, CFG])
    for a, b in ((-1, 1), (0, 3), (1, 1)):
        assert B.ods_kv_copy_pages(blk.c, a, b, FAKE, 4, None) == B.ODS_ERANGE
        assert B.ods_kv_accept(blk.c, a, b, fake_batch(), fake_draft(), FAKE, 4, FAKE, None, None) == B.ODS_ERANGE
    assert B.ods_kv_copy_pages(blk.c, 0, 2, None, 4, None) == B.ODS_EINVAL
    assert B.ods_kv_copy_pages(blk.c, 0, 2, FAKE + 4, 4, None) == B.ODS_EINVAL
    assert B.ods_kv_copy_pages(blk.c, 0, 2, FAKE, -1, None) == B.ODS_EINVAL
    assert B.ods_kv_copy_pages(blk.c, 0, 2, None, 0, None) == B.ODS_OK
    acc = lambda batch=None, draft=None, path=FAKE, cols=4, n=FAKE, out=None: B.ods_kv_accept(  # noqa: E731
        blk.c, 0, 2, batch or fake_batch(), draft or fake_draft(), path, cols, n, out, None)
    for bad in (dict(path=None), dict(n=None), dict(cols=0), dict(cols=257), dict(out=FAKE + 4), dict(path=FAKE + 4),
                dict(draft=fake_draft(row_off=None)), dict(draft=fake_draft(max_rows=0)),
                dict(batch=fake_batch(ctx_lens=None)), dict(batch=fake_batch(batch=5, ctx_lens=FAKE + 32), out=FAKE + 16)):
        assert acc(**bad) == B.ODS_EINVAL, bad
    assert acc(batch=fake_batch(batch=0)) == B.ODS_OK
    none = R.DeviceBlock([CFG], [{}], [None], 0)
    assert B.ods_kv_copy_pages(none.c, 0, 1, FAKE, 4, None) == B.ODS_EINVAL


def test_new_contexts_over_an_array_that_is_read_are_refused():
    blk, far = fake_block([CFG]), FAKE + 65536
    acc = lambda out, batch=None, draft=None, path=far, n=far: B.ods_kv_accept(  # noqa: E731
        blk.c, 0, 1, batch or fake_batch(ctx_lens=far), draft or fake_draft(row_off=far), path, 4, n, out, None)
    assert acc(FAKE, path=FAKE) == B.ODS_EINVAL
    assert acc(FAKE, n=FAKE) == B.ODS_EINVAL
    assert acc(FAKE, draft=fake_draft(row_off=FAKE)) == B.ODS_EINVAL
    assert acc(FAKE, batch=fake_batch(ctx_lens=FAKE), n=FAKE) == B.ODS_EINVAL      # in place, but over path_len
    assert "overlaps" in B.ods_last_error()


# ---------------------------------------------------------------- page bookkeeping

def check_model(k, contents, rows):
    """Holders, free list and table agree; every sequence's pages hold what the model says."""
    held = {}
    for b in range(rows):
        n = -(-int(k.tokens[b]) // 16)
        assert (k.table[b, n:] == -1).all()
        for p in k.table[b, :n]:
            held[int(p)] = held.get(int(p), 0) + 1
    refs = np.zeros(k.c.pool_pages, np.int32)
    for p, n in held.items():
        refs[p] = n
    np.testing.assert_array_equal(k._refs, refs)
    free = k._free[:k.free]
    assert sorted(free.tolist()) == [p for p in range(k.c.pool_pages) if p not in held]


def test_pages_against_a_model():
    """Random grows, trims, forks, releases and compactions; tokens are labels written through the table, copies are
    carried out on the host as kv_copy_pages would, in a shuffled order within a list."""
    rng = np.random.default_rng(5)
    rows, max_pages, pool = 6, 10, 40
    for trial in range(30):
        k = R.KvPages(pool, rows, max_pages)
        mem = np.zeros((pool, 16), np.int64)
        want = [[] for _ in range(rows)]
        label = 1

        def copies():
            for batch in k.take_copies():
                assert not set(batch[:, 0]) & set(batch[:, 1]) and len(set(batch[:, 1])) == len(batch)
                for s, d in rng.permutation(batch):
                    mem[d] = mem[s]

        for _ in range(60):
            b = int(rng.integers(rows))
            op = rng.choice(["grow", "grow", "trim", "fork", "release", "compact"])
            if op == "grow":
                new = min(max_pages * 16, int(k.tokens[b]) + int(rng.integers(0, 40)))
                try:
                    old = int(k.tokens[b])
                    k.resize(b, new)
                except B.OdsError as e:
                    assert e.status == B.ODS_ENOMEM
                    check_model(k, want, rows)
                    continue
                if rng.random() < 0.5:
                    copies()
                    for t in range(old, new):
                        mem[k.table[b, t // 16], t % 16] = label
                        want[b].append(label)
                        label += 1
                else:  # a second operation before the copies: write only after them
                    c = int(rng.integers(rows))
                    if c != b and not k.tokens[c] and len(want[b]) == old == new:
                        k.fork(b, c)
                        want[c] = list(want[b])
                    copies()
                    for t in range(old, new):
                        mem[k.table[b, t // 16], t % 16] = label
                        want[b].append(label)
                        label += 1
            elif op == "trim":
                new = int(rng.integers(0, int(k.tokens[b]) + 1))
                k.resize(b, new)
                del want[b][new:]
            elif op == "fork":
                c = int(rng.integers(rows))
                if c != b and not k.tokens[c]:
                    k.fork(b, c)
                    want[c] = list(want[b])
            elif op == "release":
                k.release(b)
                want[b] = []
            else:
                k.compact(None if rng.random() < 0.7 else 2)
                copies()
            check_model(k, want, rows)
            for r in range(rows):
                assert [int(mem[k.table[r, t // 16], t % 16]) for t in range(int(k.tokens[r]))] == want[r]
        k.compact()
        copies()
        n = pool - k.free
        assert k.table.max() < n


def test_copies_that_meet_are_ordered():
    """A page freed by one operation and written by the next copy: two lists, the first one's read comes first."""
    k = R.KvPages(4, 3, 2)
    k.resize(0, 20)                     # pages 0, 1
    k.fork(0, 1)
    k.resize(1, 21)                     # row 1's own page: 1 -> 2
    k.release(0)                        # pages 1 free again (0 still held by row 1)
    k.fork(1, 2)
    k.resize(2, 22)                     # row 2's own page: 2 -> 1
    assert [c.tolist() for c in k.take_copies()] == [[[1, 2]], [[2, 1]]]
    assert k.take_copies() == []


def test_pages_adopt_a_table_and_refuse():
    ctx = np.array([20, 16, 1, 33], np.int32)
    t = np.zeros((4, 4), np.int32)
    assert B.ods_kv_alloc(12, ctx, 4, 3, 4, t) == B.ODS_OK
    k = R.KvPages(12, 4, 4, table=t, tokens=ctx)
    assert k.free == 12 - 7
    check_model(k, None, 4)
    before = k.table.copy(), k._refs.copy(), k.free
    for call in (lambda: k.resize(0, 65), lambda: k.resize(0, -1), lambda: k.fork(0, 1), lambda: k.fork(0, 0)):
        with pytest.raises((B.OdsError, ValueError)):
            call()
    k.tokens[0] = 40                    # not what the row holds
    with pytest.raises(B.OdsError):
        k.resize(0, 41)
    k.tokens[0] = 20
    one, pair = k.table[0], np.zeros(2, np.int32)
    assert B.lib.ods_pages_resize(C.byref(k.c), one.ctypes.data, 4, 20, 30, None, None) == B.ODS_EINVAL
    assert B.lib.ods_pages_resize(None, one.ctypes.data, 4, 20, 30, pair.ctypes.data, pair.ctypes.data) == B.ODS_EINVAL
    assert B.ods_pages_init(k.c, np.array([[12]], np.int32)) == B.ODS_ERANGE
    bad = k.table.copy()
    bad[0, 0] = -1                      # not the holders
    assert B.ods_pages_compact(k.c, bad, np.zeros((4, 2), np.int32))[0] == B.ODS_EINVAL
    loose = np.array([11, -1], np.int32) if 11 not in k.table else np.array([int(k._free[0]), -1], np.int32)
    assert B.ods_pages_release(k.c, loose) == B.ODS_EINVAL
    np.testing.assert_array_equal(k.table, before[0])
    np.testing.assert_array_equal(k._refs, before[1])
    assert k.free == before[2]
    n = np.zeros(1, np.int32)
    k.c.n_free = 13
    assert B.lib.ods_pages_fork(C.byref(k.c), one.ctypes.data, n.ctypes.data, 1, 1) == B.ODS_EINVAL


@pytest.mark.skipif(shutil.which(CXX) is None, reason="no host C++ compiler")
def test_host_sources_are_clean_under_asan_and_ubsan(tmp_path):
    exe, src = tmp_path / "draft_check", os.path.join(ROOT, "paper_2609_14237_amd", "csrc")
    cmd = [CXX, "-std=c++17", "-g", "-O1", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
           os.path.join(ROOT, "include"), *(os.path.join(src, f) for f in ("ods_host.cpp", "ods_draft.cpp", "ods_pages.cpp")),
           os.path.join(ROOT, "tests", "host", "draft_check.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "draft_check OK" in r.stdout
