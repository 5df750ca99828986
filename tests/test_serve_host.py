"""Host-side checks, without a GPU, of normalised heads, shared prefixes and the verification of drafted tokens: every
refusal (all return before anything is enqueued), groups found in page tables, workspace sizes."""
import ctypes as C
import os
import shutil
import subprocess
from dataclasses import replace

import numpy as np
import pytest
import torch

import serve_ref as S
import workloads as W

B = pytest.importorskip("paper_2609_14237_amd.binding")
from paper_2609_14237_amd import runtime as R  # noqa: E402
from test_draft_host import CFG, CXX, FAKE, ROOT, fake_batch, fake_block, fake_state, rope_struct  # noqa: E402

FAR = FAKE + (1 << 20)


def gains(q=FAKE, k=FAKE, eps=1e-6):
    return B.ods_head_norm(q, k, eps)


def test_head_rows_refusals():
    r = rope_struct()

    def call(norm=gains(), **k):
        f = dict(r=r, axis=None, n_axes=1, x=FAKE, xs=512, y=FAR, ys=512, rows=4, n_q=2, n_k=1, pos=FAKE)
        f.update(k)
        return B.ods_head_rows(f["r"], norm, f["axis"], f["n_axes"], f["x"], f["xs"], f["y"], f["ys"], f["rows"], f["n_q"], f["n_k"],
                               f["pos"], None)

    assert B.lib.ods_head_rows(None, None, None, 1, FAKE, 512, FAR, 512, 4, 2, 1, FAKE, None) == B.ODS_EINVAL
    for bad in (dict(x=None), dict(y=None), dict(pos=None), dict(pos=FAKE + 2), dict(x=FAKE + 8), dict(y=FAR + 2), dict(rows=-1),
                dict(n_q=-1), dict(n_k=-1), dict(n_q=2 ** 31 - 1, n_k=1), dict(xs=376), dict(ys=385), dict(n_axes=0),
                dict(n_axes=B.ROPE_AXES + 1, axis=FAKE), dict(n_axes=2), dict(axis=FAKE + 2), dict(r=rope_struct(freqs=None)),
                dict(y=FAKE + 16), dict(norm=gains(eps=-1.0)), dict(norm=gains(eps=float("nan"))), dict(norm=gains(eps=float("inf"))),
                dict(norm=gains(q=None)), dict(norm=gains(k=None)), dict(norm=gains(q=FAKE + 8)), dict(norm=gains(k=FAKE + 2))):
        assert call(**bad) == B.ODS_EINVAL, bad
    assert call(r=rope_struct(head_dim=264)) == B.ODS_EUNSUPPORTED
    assert call(rows=0, x=None) == B.ODS_OK and call(n_q=0, n_k=0, norm=gains(None, None)) == B.ODS_OK
    assert call(rows=0, n_k=0, norm=gains(k=None)) == B.ODS_OK and call(rows=0, n_q=0, norm=gains(q=None)) == B.ODS_OK


def draft(norm=None, shared=None, **kw):
    f = dict(rows=8, max_rows=4, row_off=FAKE, depth=FAKE, mask=FAKE)
    f.update(kw)
    return B.ods_draft(f["rows"], f["max_rows"], f["row_off"], f["depth"], f["mask"], None,
                       None if norm is None else C.cast(norm, C.POINTER(B.ods_head_norm)), None if shared is None else C.pointer(shared))


def test_norms_and_groups_of_drafted_rows_are_refused():
    blk = fake_block([CFG, replace(CFG, window=40)])
    run = lambda a, b, d, batch=None, st=None: B.ods_run_draft(blk.c, a, b, batch or fake_batch(), d, st or fake_state(), None)  # noqa: E731
    for bad in (gains(q=None), gains(k=None), gains(eps=-1e-9), gains(k=FAKE + 8)):
        two = (B.ods_head_norm * 2)(gains(), bad)
        assert run(12, 13, draft(norm=two)) == B.ODS_EINVAL
        assert run(0, 20, draft(norm=two)) == B.ODS_EINVAL
    for bad in ((-1, FAKE, FAKE), (3, FAKE, FAKE), (2, None, FAKE), (2, FAKE, None), (1, FAKE + 8, FAKE), (1, FAKE, FAKE + 4)):
        assert run(4, 5, draft(shared=B.ods_shared(*bad))) == B.ODS_EINVAL, bad
    assert run(4, 5, draft(rows=5000, max_rows=1, shared=B.ods_shared(4096, FAKE, FAKE)), fake_batch(batch=4096)) == B.ODS_EUNSUPPORTED
    # n_kv * query tiles of 2^20 rows * pages of a table this wide: the kernel's unit index
    wide = fake_block([replace(CFG, n_q=32, n_kv=2)])
    assert B.ods_run_draft(wide.c, 4, 5, fake_batch(max_pages=1 << 14), draft(rows=1 << 20, max_rows=2, shared=B.ods_shared(1, FAKE, FAKE)),
                           fake_state(), None) == B.ODS_EUNSUPPORTED
    long, one = fake_batch(max_pages=1 << 14), B.ods_shared(1, FAKE, FAKE)
    assert B.ods_draft_workspace_bytes(blk.c, long, draft(shared=one)) > B.ods_draft_workspace_bytes(blk.c, long, draft())
    assert B.ods_draft_workspace_bytes(blk.c, fake_batch(), draft(shared=one)) == B.ods_draft_workspace_bytes(blk.c, fake_batch(), draft())
    assert run(4, 5, draft(shared=B.ods_shared(1, FAKE, FAKE)), st=fake_state(ws_bytes=8 * 4 * 66 * 4)) == B.ODS_ENOMEM
    assert B.ods_draft_workspace_bytes(blk.c, fake_batch(), draft(shared=B.ods_shared(3, FAKE, FAKE))) == 0
    # nothing to do
    assert run(0, 20, draft(rows=0, row_off=None, shared=B.ods_shared(2, None, None))) == B.ODS_OK


@pytest.mark.parametrize("n_q,n_kv,hd", [(4, 2, 64), (32, 8, 128), (16, 1, 128), (3, 3, 64)])
def test_a_workspace_for_the_widest_serves_all_narrower(n_q, n_kv, hd):
    blk = fake_block([replace(CFG, n_q=n_q, n_kv=n_kv, head_dim=hd)])
    size = lambda b, pages, rows, most, n: B.ods_draft_workspace_bytes(  # noqa: E731
        blk.c, fake_batch(batch=b, max_pages=pages), draft(rows=rows, max_rows=most, shared=None if n is None else B.ods_shared(n, FAKE, FAKE)))
    whole = size(64, 512, 64 * 16, 16, 7)
    for b in (1, 3, 20, 64):
        for pages in (1, 30, 512):
            for most in (1, 2, 5, 16):
                for n in (None, 0, 1, 2, b):
                    for rows in (1, b * most):
                        if n is None or n <= b:
                            assert 0 < size(b, pages, rows, most, n) <= whole, (b, pages, most, n, rows)


def test_groups_of_a_table():
    t = lambda *rows: np.array([list(r) + [-1] * (6 - len(r)) for r in rows], np.int32)  # noqa: E731

    def found(table, tokens):
        n, off, tok = len(tokens), np.full(len(tokens) + 1, 99, np.int32), np.full(max(len(tokens), 1), 99, np.int32)
        st, k = B.ods_pages_shared(table, np.array(tokens, np.int32), off, tok)
        assert st == B.ODS_OK
        return off[:k + 1].tolist(), tok[:k].tolist()

    assert found(t((1, 2, 3), (1, 2, 4), (1, 2)), [48, 40, 32]) == ([0, 3], [32])
    assert found(t((1, 2, 3), (1, 2, 4), (1, 2)), [48, 40, 31]) == ([0, 3], [16])             # two save two pages, three of one page no fewer
    assert found(t((1, 2, 3), (1, 2, 3), (1, 9)), [48, 48, 32]) == ([0, 2, 3], [48, 0])       # three save fewer than two
    assert found(t((1,), (2,), (3,)), [16, 16, 16]) == ([0, 3], [0])
    assert found(t((1,), (2,), (2, 5), (6,), (7,)), [16, 16, 20, 3, 0]) == ([0, 1, 3, 5], [0, 16, 0])
    assert found(t((1, 2, 3, 4, 5), (1, 2, 3, 4, 5), (1,), (1,)), [80, 80, 16, 16]) == ([0, 2, 4], [80, 16])
    assert found(t((-1,), (-1,)), [16, 16]) == ([0, 2], [0])
    assert found(np.zeros((0, 6), np.int32), []) == ([0], [])
    one = np.zeros((1, 6), np.int32)
    off, tok = np.zeros(2, np.int32), np.zeros(1, np.int32)
    for tokens in (-1, 97):
        assert B.ods_pages_shared(one, np.array([tokens], np.int32), off, tok)[0] == B.ODS_EINVAL
    n = C.c_int32()
    for i in range(5):
        a = [one.ctypes.data, 1, 6, off.ctypes.data, off.ctypes.data, tok.ctypes.data, C.addressof(n)]
        a[(0, 3, 4, 5, 6)[i]] = None
        assert B.lib.ods_pages_shared(*a) == B.ODS_EINVAL
    assert B.lib.ods_pages_shared(one.ctypes.data, -1, 6, off.ctypes.data, off.ctypes.data, tok.ctypes.data, C.addressof(n)) == B.ODS_EINVAL


def test_groups_of_forks():
    k = R.KvPages(pool_pages=100, rows=5, max_pages=20)
    k.resize(0, 100)
    for b in (1, 2):
        k.fork(0, b)
        k.resize(b, 101 + b)
    k.resize(3, 40)
    off, tokens = k.shared()
    assert off.tolist() == [0, 3, 5] and tokens.tolist() == [96, 0]
    with pytest.raises(ValueError):
        R.SharedPrefix(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        R.SharedPrefix(torch.zeros(3), torch.zeros(2, dtype=torch.int32))


def verify(**kw):
    f = dict(vocab=100, dtype=0, target=FAKE, target_stride=100, proposal=None, proposal_stride=0, tokens=FAKE, parent=FAKE, accept_u=FAKE,
             next_u=FAKE, path_cols=4, path=FAKE, path_len=FAKE, next_token=FAKE, ws=FAKE, ws_bytes=1 << 30)
    f.update(kw)
    return B.ods_verify(*[f[n] for n, _ in B.ods_verify._fields_])


def test_verify_refusals():
    run = lambda d=None, batch=2, **kw: B.ods_draft_verify(batch, d or draft(), verify(**kw), None)  # noqa: E731
    assert B.lib.ods_draft_verify(2, None, C.byref(verify()), None) == B.ODS_EINVAL
    assert B.lib.ods_draft_verify(2, C.byref(draft()), None, None) == B.ODS_EINVAL
    for bad in (dict(vocab=0), dict(vocab=B.VERIFY_MAX_VOCAB + 1, target_stride=1 << 30), dict(dtype=2), dict(dtype=-1), dict(target=None),
                dict(target=FAKE + 2), dict(dtype=1, target=FAKE + 1), dict(target_stride=99), dict(target_stride=1 << 61),
                dict(proposal=FAKE, proposal_stride=99), dict(proposal=FAKE + 1, proposal_stride=100), dict(path_cols=0), dict(path_cols=257),
                dict(ws=None), dict(ws=FAKE + 8),
                *(d for n in ("tokens", "parent", "accept_u", "next_u", "path", "path_len", "next_token") for d in ({n: None}, {n: FAKE + 2}))):
        assert run(**bad) == B.ODS_EINVAL, bad
    for d in (dict(rows=-1), dict(max_rows=0), dict(max_rows=257), dict(row_off=None), dict(row_off=FAKE + 4)):
        assert run(draft(**d)) == B.ODS_EINVAL, d
    assert run(batch=-1) == B.ODS_EINVAL and run(batch=4097) == B.ODS_EUNSUPPORTED
    assert run(draft(rows=(1 << 20) + 1)) == B.ODS_EUNSUPPORTED
    need = B.ods_verify_workspace_bytes(2, 100)
    assert need > 0 and run(ws_bytes=need - 1) == B.ODS_ENOMEM
    assert run(batch=0, target=None, path=None, ws=None) == B.ODS_OK
    for b, v in ((-1, 5), (4097, 5), (1, 0), (1, B.VERIFY_MAX_VOCAB + 1)):
        assert B.ods_verify_workspace_bytes(b, v) == 0
    assert B.ods_verify_workspace_bytes(3, 5000) <= B.ods_verify_workspace_bytes(3, 5001) <= B.ods_verify_workspace_bytes(4, 9000)


def test_python_side_refusals():
    i32, f32, bf = torch.int32, torch.float32, torch.bfloat16
    z = lambda *s, dt=i32: torch.zeros(*s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError):
        R.HeadNorm(z(64, dt=f32))
    with pytest.raises(ValueError):
        R.HeadNorm(z(64, dt=bf), z(128, dt=bf))
    for sections in ((16, 15), (16, 17), (33, -1), (), (4,) * 8 + (0,)):
        with pytest.raises(ValueError):
            R.Rope(64, sections=sections, device="cpu")
    with pytest.raises(ValueError):
        R.Rope(64, sections=(16, 16), order="other", device="cpu")
    blk = fake_block([CFG])
    batch = R.DeviceBatch(z(2), z(2, 4))
    for norm in ([], [R.HeadNorm(z(128, dt=bf), z(128, dt=bf))]):
        with pytest.raises(ValueError):
            R.run_draft(blk, 2, 5, batch, R.DeviceDraft(z(3), z(8), z(8, dt=torch.int64), max_rows=64, norm=norm), R.ods_state())
    for args in ((-1, 4, 5), (4097, 4, 100), (0, 4, 0), (4, 0, 100), (4, 257, 100), (4, 4, B.VERIFY_MAX_VOCAB + 1)):
        with pytest.raises(ValueError):
            R.DraftVerifier(*args, device="cpu")
    v, d = R.DraftVerifier(2, 4, 100, device="cpu"), R.DeviceDraft(z(3), z(8), z(8, dt=torch.int64), max_rows=4)
    good = dict(tokens=z(8), parent=z(8), target=z(8, 100, dt=f32), accept_u=z(8, dt=f32), next_u=z(2, dt=f32))
    for bad in (dict(tokens=z(7)), dict(parent=z(8, dt=torch.int64)), dict(target=z(8, 101, dt=f32)), dict(target=z(8, 100, dt=torch.float16)),
                dict(target=z(7, 100, dt=f32)), dict(target=z(100, 8, dt=f32).T), dict(accept_u=z(8)), dict(next_u=z(8, dt=f32)),
                dict(proposal=z(8, 99, dt=f32)), dict(proposal=z(8, 100, dt=bf)), dict(tokens=z(16)[::2])):
        with pytest.raises(ValueError):
            v.run(d, **{**good, **bad})
    with pytest.raises(ValueError):
        v.run(R.DeviceDraft(z(4), z(8), z(8, dt=torch.int64), max_rows=4), **{**good, "next_u": z(3, dt=f32)})


@pytest.mark.parametrize("sections,order", [((16, 24, 24), "blocks"), ((16, 24, 24), "cyclic"), ((0, 64), "cyclic"), ((64,), "blocks"),
                                            ((1, 2, 3, 4, 5, 6, 7, 36), "cyclic")])
@pytest.mark.parametrize("own", [False, True])
def test_axes_and_their_frequencies(sections, order, own):
    r = R.Rope(128, theta=5e5, sections=sections, order=order, own_freqs=own, device="cpu")
    axis, f = S.section_freqs(sections, order, 5e5, 128, own)
    np.testing.assert_array_equal(r.axis.numpy(), axis)
    np.testing.assert_allclose(r.freqs.numpy(), f, rtol=1e-13)


def test_the_reference_keeps_the_targets_distribution():
    """The definition itself, by exact enumeration over fine random numbers: a chain of one draft, vocabulary of three."""
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.2, 0.5, 0.3])
    n, got = 200, np.zeros(3)
    grid = (np.arange(n) + 0.5) / n
    for x in range(3):
        for u in grid:
            path, lens, _ = S.verify([0, 2], 2, 2, [0, x], [-1, 0], np.stack([p, p]), np.stack([q, q]), [0, u], [0.5], 2, 3)
            if lens[0] == 2:
                got[x] += q[x] / n
            else:
                w = np.maximum(p - q, 0)
                got += q[x] / n * w / w.sum()
    np.testing.assert_allclose(got, p, atol=1.0 / n)


@pytest.mark.skipif(shutil.which(CXX) is None, reason="no host compiler")
def test_host_parts_under_the_sanitizers(tmp_path):
    src, exe = os.path.join(ROOT, "paper_2609_14237_amd", "csrc"), tmp_path / "serve_check"
    cmd = [CXX, "-std=c++17", "-g", "-O1", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
           *(os.path.join(src, f) for f in ("ods_host.cpp", "ods_draft.cpp", "ods_pages.cpp", "ods_verify.cpp")),
           os.path.join(ROOT, "tests", "host", "serve_check.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1"))
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "serve_check OK" in r.stdout
