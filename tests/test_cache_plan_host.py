"""The plan that deals out the tiles of an attention call, compiled for the host: numbers of tiles at the library's limits."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <cstdio>
#include <vector>
#include "pkv_cache_attend.cuh"
int main() {
  const long long cases[][3] = {{1024, 2097151, 1}, {1024, 2097151, 64}, {128, 16777215, 8}, {3, 1, 2}};   // sequences, tiles of each, units
  for (const auto& c : cases) {
    std::vector<int32_t> off(c[0] + 1);
    for (long long s = 0; s <= c[0]; ++s) off[s] = static_cast<int32_t>(s * c[1]);
    pkv::CaPlan plan{};
    plan.per_seq = static_cast<int>(c[2]);
    for (long long s = 0; s <= c[0]; ++s) {
      const long long want = (s * c[1] + pkv::kCaStart * s) * c[2], got = plan.ahead(off.data(), static_cast<int>(s));
      if (got != want) { std::printf("%lld tiles x %lld: %lld ahead of sequence %lld, not %lld\n", c[1], c[2], got, s, want); return 1; }
    }
  }
  return 0;
}
"""


@pytest.mark.skipif(shutil.which(os.environ.get("NVCC", "nvcc")) is None, reason="needs nvcc")
def test_tiles_ahead_of_a_sequence_are_counted_in_64_bits(tmp_path):
    (tmp_path / "plan.cu").write_text(SOURCE)
    subprocess.check_call([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2406_02069_b200", "csrc"), "-o", str(tmp_path / "plan"), str(tmp_path / "plan.cu")])
    run = subprocess.run([str(tmp_path / "plan")], stdout=subprocess.PIPE, universal_newlines=True)
    assert run.returncode == 0, run.stdout
