"""The record of outputs that calls of the library may still be writing, compiled for the host: what it must not lose, and what it
lets go of."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <cstdio>
#include "pkv_host.cuh"
using namespace pkv;
static int failed = 0;
static StreamKey stream(uintptr_t i, uint64_t capture = 0) { return StreamKey{reinterpret_cast<cudaStream_t>(0x100000 + 64 * i), -1, 0, capture}; }
static void* at(uintptr_t a) { return reinterpret_cast<void*>(a); }
static bool known(uintptr_t lo, uintptr_t hi, uint64_t capture = 0) { return g_outputs.overlaps(capture, lo, hi); }
static void want(bool ok, const char* what) { if (!ok) { std::printf("%s\n", what); failed = 1; } }
static void note_launch(const StreamKey& k) { g_outputs.launched(k); }
static void note_output(const void* p, size_t n, const StreamKey& k) { g_outputs.wrote(k, {{p, n}}); }
static void launch(const StreamKey& k, int n = 1) { for (int i = 0; i < n; ++i) note_launch(k); }
int main() {
  const StreamKey a = stream(1), b = stream(2);
  note_launch(a);
  note_output(at(0x10000), 0x100, a);
  want(known(0x10000, 0x10001) && known(0x100ff, 0x20000) && known(0, 0x10001), "an output is known");
  want(!known(0x10100, 0x20000) && !known(0, 0x10000), "its neighbours are not");
  for (int i = 0; i < 1000; ++i) {         // appends of another stream, three outputs each
    note_launch(b);
    for (uintptr_t o = 0; o < 3; ++o) note_output(at(0x1000000 + 0x1000 * (3 * i + o)), 0x100, b);
  }
  want(known(0x10000, 0x10100), "launches on another stream say nothing about it");
  want(known(0x1000000 + 0x1000 * 2999, 0x1000000 + 0x1000 * 2999 + 1), "the other stream's last output");
  want(known(0x1000000 + 0x1000 * (3 * 999 - 3 * 126), 0x1000000 + 0x1000 * (3 * 999 - 3 * 126) + 1), "and those of the launches that may be with it");
  want(!known(0x1000000, 0x1000000 + 0x1000 * 2000), "not those of long ago");
  for (int i = 0; i < 126; ++i) {          // the same cache again and again on its own stream
    note_launch(a);
    for (uintptr_t o = 0; o < 3; ++o) note_output(at(0x40000 + 0x1000 * o), 0x800, a);
  }
  want(known(0x10000, 0x10100), "126 launches behind it");
  launch(a, 2);
  want(!known(0x10000, 0x10100), "128 launches behind it: complete");
  want(known(0x40000, 0x40001) && known(0x42000, 0x42001), "what was written again is as young as its last writer");
  launch(a, 128);
  want(!known(0x40000, 0x43000), "and lets go then");
  // one range within another, in either order
  note_launch(a);
  note_output(at(0x50000), 0x1000, a);
  launch(a, 100);
  note_output(at(0x50400), 0x100, a);
  launch(a, 60);
  want(known(0x50400, 0x50500) && !known(0x50000, 0x50400), "a part is written again: the rest is older");
  note_output(at(0x50000), 0x1000, a);
  launch(a, 100);
  want(known(0x50000, 0x50001) && known(0x50fff, 0x51000), "the whole again");
  // captures: launches that are captured are not behind anything that runs, and a capture looks at its own outputs only
  note_launch(a);
  note_output(at(0x60000), 0x100, a);
  launch(stream(1, 7), 500);
  want(known(0x60000, 0x60100), "captured launches are not behind it");
  note_output(at(0x68000), 0x100, stream(1, 7));
  note_launch(stream(2, 7));
  note_output(at(0x69000), 0x100, stream(2, 7));
  want(known(0x68000, 0x68100, 7) && known(0x69000, 0x69100, 7), "outputs of a capture, on both of its streams");
  want(!known(0x68000, 0x69100) && !known(0x68000, 0x69100, 8) && !known(0x60000, 0x60100, 7), "are nobody else's");
  note_launch(stream(1, 8));
  want(!known(0x68000, 0x68100, 8) && known(0x69000, 0x69100, 7), "another capture on the stream starts with nothing");
  launch(a, 128);
  want(!known(0x60000, 0x60100), "launches that run are");
  // more streams than there is room for: nothing is lost
  for (uintptr_t s = 10; s < 300; ++s) {
    note_launch(stream(s));
    note_output(at(0x80000000ull + s * 0x10000), 0x100, stream(s));
  }
  for (uintptr_t s = 10; s < 300; ++s) want(known(0x80000000ull + s * 0x10000, 0x80000000ull + s * 0x10000 + 1), "an output of one of many streams");
  want(!known(0x1000, 0x50000), "below all of them (a range of its own holds what had to make room, stream a's 0x50000 the lowest)");
  note_output(nullptr, 64, a);
  note_output(at(64), 0, a);
  want(!known(0, 0x100), "nothing written");
  return failed;
}
"""


@pytest.mark.skipif(shutil.which(os.environ.get("NVCC", "nvcc")) is None, reason="needs nvcc")
def test_outputs_are_known_until_they_are_complete(tmp_path):
    (tmp_path / "outputs.cu").write_text(SOURCE)
    subprocess.check_call([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2406_02069_b200", "csrc"), "-o", str(tmp_path / "outputs"), str(tmp_path / "outputs.cu")])
    run = subprocess.run([str(tmp_path / "outputs")], stdout=subprocess.PIPE, universal_newlines=True)
    assert run.returncode == 0, run.stdout
