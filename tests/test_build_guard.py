"""The build refuses kernels that spill vector registers, of every source."""
import os
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
