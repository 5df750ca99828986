"""The build refuses kernels that spill vector registers, of every source; what a kernel holds that one form of a call does not
need is not held for the others."""
import os
import re
import shutil

import pytest

from paper_2609_14237_amd import build

# 96 floats a lane, all in use across a barrier, where a lane has 64 registers
SPILLS = r"""
#include <hip/hip_runtime.h>
extern "C" __global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(8))) void k(float *x) {
  float v[96];
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int i = 0; i < 96; ++i) v[i] = x[i * 512 + threadIdx.x + r];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 96; ++i) x[((i * 37 + 11) % 96) * 512 + threadIdx.x] = v[i] * v[(i + 1) % 96];
    __syncthreads();
  }
}
"""
FITS = r"""
#include <hip/hip_runtime.h>
extern "C" __global__ void k(float *x) { x[threadIdx.x] *= 2.f; }
"""


pytestmark = pytest.mark.skipif(shutil.which(build.HIPCC) is None, reason="no hipcc")


def test_others_are_built(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path))
    (tmp_path / "k_tree.hip").write_text(FITS)
    assert os.path.exists(build._compile("k_tree.hip"))


@pytest.mark.parametrize("name", sorted(s for s in build.SOURCES if s.endswith(".hip")))
def test_spills_are_refused(name, tmp_path, monkeypatch):
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path))
    (tmp_path / name).write_text(SPILLS)
    with pytest.raises(RuntimeError, match="spills"):
        build._compile(name)


def test_rotations_without_a_norm_hold_nothing_for_one():
    """LDS of the drafted rows' RoPE and append: a row's cosines and sines, and what the norm exchanges only where there is one."""
    usage = os.path.join(build.BUILD_DIR, "k_tree.hip.o.usage")
    if not os.path.exists(usage):
        os.makedirs(build.BUILD_DIR, exist_ok=True)
        build._compile("k_tree.hip")
    held = {}
    for part in re.split(r"Function Name: ", open(usage).read())[1:]:
        if "draft_rope_append_kernel" in part.split()[0]:
            held[part.split()[0]] = int(re.search(r"LDS Size \[bytes/block\]: (\d+)", part).group(1))
    assert sorted(held.values()) == [2 * 128 * 4, 2 * 128 * 4 + 8 * 256 * 4]
