"""Which tiles of a walk are read whole (CPU): compiled from the library's header, under the sanitizer for
undefined arithmetic."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")

SOURCE = r"""
#include <cstdio>
#include <random>
#include "walk.h"
using namespace medha;
int main() {
  std::mt19937 rng(11);
  auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
  for (int it = 0; it < 20000; ++it) {
    const int span = upto(140);
    const int a = upto(3) ? upto(900) : INT32_MAX - 1 - span - upto(80), b = a + span;
    Window win;
    win.keys = upto(8) ? 1 + upto(300) : 1 + upto(3);
    win.sinks = upto(3) ? upto(30) : upto(300);
    const KeyWalk w = make_walk(a, b, win, 64);
    const WholeTiles whole(w);
    for (int i = 0; i < w.n; ++i) {
      const int64_t t = w.tile(i), lo = w.first_tokens(i) ? 0 : w.lo, end = w.first_tokens(i) ? w.first : w.end;
      const bool want = t * 64 >= lo && (t + 1) * 64 <= end;
      const bool got = whole.holds(w.first_tokens(i) ? ~(int)t : (int)t);
      if (got != want) return std::printf("[%d, %d] window %d, %d first: tile %d is %d\n", a, b, win.keys, win.sinks, (int)t, got), 1;
    }
  }
  std::printf("ok\n");
}
"""


def test_whole_tiles(tmp_path):
    src, exe = tmp_path / "whole.hip", str(tmp_path / "whole")
    src.write_text(SOURCE)
    res = subprocess.run([HIPCC, "-O1", "-g", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17",
                          "-Xarch_host", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                          "-I", os.path.join(ROOT, "paper_2409_17264_amd", "csrc"), str(src), "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "ok" in run.stdout, run.stdout + run.stderr[-3000:]
