"""Host checks, without a GPU, of what a drafted range's validation costs and how its workspace is sized, under the CPU
sanitizers."""
import os
import shutil
import subprocess

import pytest

import workloads as W

B = pytest.importorskip("paper_2609_14237_amd.binding")
from test_draft_host import fake_batch, fake_block, fake_draft, fake_state  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = os.environ.get("CXX", "g++")


@pytest.mark.skipif(shutil.which(CXX) is None, reason="no host C++ compiler")
def test_sizes_of_drafted_ranges(tmp_path):
    exe, src = tmp_path / "draft_sizes_check", os.path.join(ROOT, "paper_2609_14237_amd", "csrc")
    cmd = [CXX, "-std=c++17", "-g", "-O1", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
           os.path.join(ROOT, "include"), *(os.path.join(src, f) for f in ("ods_host.cpp", "ods_draft.cpp", "ods_pages.cpp")),
           os.path.join(ROOT, "tests", "host", "draft_sizes_check.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "draft_sizes_check OK" in r.stdout


@pytest.mark.parametrize("cfg,batch,pages", [
    (W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512), 32, 256),
    (W.LayerCfg(hidden=256, n_q=4, n_kv=2, head_dim=64, ffn=512), 64, 40),
    (W.BY_NAME["dense8b_b64"].layers[0], 32, 256)])
def test_a_workspace_of_wide_trees_serves_narrow_ones(cfg, batch, pages):
    """ods_draft_workspace_bytes never shrinks with the rows of a sequence."""
    blk = fake_block([cfg])
    sizes = [B.ods_draft_workspace_bytes(blk.c, fake_batch(batch=batch, max_pages=pages), fake_draft(rows=batch * m, max_rows=m))
             for m in range(1, 257)]
    assert sizes[0] > 0 and sizes == sorted(sizes)


def test_rows_that_can_only_be_padding_are_refused():
    """4096 sequences of 256 rows are 2^20; the row-wise operators' launches end at 2^24 workgroups."""
    blk, most = fake_block([W.LayerCfg(hidden=64, n_q=1, n_kv=1, head_dim=64, ffn=64)]), 1 << 20
    for rows in (most + 1, 1 << 24, 1 << 30):
        for ops in ((0, 1), (2, 5), (5, 10)):
            assert B.ods_run_draft(blk.c, *ops, fake_batch(), fake_draft(rows=rows, row_off=None), fake_state(resid=None, qkv=None),
                                   None) == B.ODS_EUNSUPPORTED
        assert B.ods_draft_workspace_bytes(blk.c, fake_batch(), fake_draft(rows=rows)) == 0
        assert B.ods_kv_accept(blk.c, 0, 1, fake_batch(), fake_draft(rows=rows), None, 4, None, None, None) == B.ODS_EUNSUPPORTED
    assert B.ods_run_draft(blk.c, 5, 10, fake_batch(), fake_draft(rows=most), fake_state(resid=None), None) == B.ODS_EINVAL
    assert B.ods_draft_workspace_bytes(blk.c, fake_batch(), fake_draft(rows=most)) > 0
