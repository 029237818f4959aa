"""Plans of windowed calls and calls over the 8-bit cache (CPU), compiled from the library's own planner: the
launches of two small workgroups to a compute unit that the GPU tests mean to run, and least workspaces."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CSRC = os.path.join(ROOT, "paper_2409_17264_amd", "csrc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")

SOURCE = r"""
#include <cstdio>
#include "planner.h"
using namespace medha;
int main() {
  // the calls of test_workgroups_in_pairs: 32/8 heads, d 128
  struct { bool fp8; int prefix, chunk, window; } pairs[] = {
      {true, 6000, 200, 0}, {true, 9000, 130, 0}, {true, 9007, 130, 8000}, {false, 9007, 130, 8000},
      {false, 6011, 200, 6000}};
  for (const auto& c : pairs) {
    Window w;
    if (c.window) w = Window{c.window, 5};
    const SeqInput s{0, 0, 0, c.chunk, c.prefix};
    const Plan p = make_plan(&s, 1, 32, 8, 128, 256, SIZE_MAX, w, c.fp8);
    std::printf("%d %d %d %d: paired %d, %d rows, %d slots\n", c.fp8, c.prefix, c.chunk, c.window, p.rows.paired,
                p.rows.shape.rows_per_wg, p.rows.n_slots);
    if (!p.rows.paired || p.rows.shape.rows_per_wg != 128 || p.rows.n_slots <= 256) return 1;
  }
  // scratch that a plan can do without
  for (bool fp8 : {false, true}) {
    const Window w{4500, 3};
    const SeqInput s[2] = {{0, 0, 0, 64, 5000}, {0, 64, 64, 1, 4000}};
    const Plan full = make_plan(s, 2, 8, 1, 128, 256, SIZE_MAX, w, fp8);
    if (full.min_bytes >= full.bytes) return 2;
    const Plan least = make_plan(s, 2, 8, 1, 128, 256, full.min_bytes, w, fp8);
    if (least.bytes > full.min_bytes || least.part_rows == 0) return 3;
  }
  std::printf("ok\n");
}
"""


def test_plans(tmp_path):
    src, exe = tmp_path / "plans.hip", str(tmp_path / "plans")
    src.write_text(SOURCE)
    res = subprocess.run([HIPCC, "-O1", "--offload-arch=gfx950", "-std=c++17", "-Wno-inline-asm", "-Xclang",
                          "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", CSRC, "-I",
                          os.path.join(ROOT, "include"), str(src), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "ok" in run.stdout, run.stdout + run.stderr
