"""Windows on the host (CPU): the walk of a window's keys and the plans made of it, compiled from the
library's own headers, and the host code of their entry points under the sanitizers."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CSRC = os.path.join(ROOT, "paper_2409_17264_amd", "csrc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
FLAGS = ["--offload-arch=gfx950", "-std=c++17", "-Wno-inline-asm", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-I", CSRC, "-I", os.path.join(ROOT, "include")]

WALKS = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "planner.h"
using namespace medha;
static std::mt19937 rng(5);
static int upto(int n) { return (int)(rng() % (unsigned)n); }
#define CHECK(x) do { if (!(x)) { std::printf("%s: %s\n", what, #x); return 1; } } while (0)

static Window window() {
  Window w;
  if (upto(10) == 0) return w;
  w.keys = upto(5) ? 1 + upto(500) : 1 + upto(3);
  w.sinks = upto(3) ? upto(20) : upto(600);
  return w;
}

// Every row is shown each key that it sees once and no other; what a visit reads is seen by some row;
// visits that need no mask show every row everything.
static int walks() {
  const char* what = "walks";
  for (int it = 0; it < 20000; ++it) {
    const int T = upto(2) ? 64 : 32, a = upto(700), b = a + upto(130);
    const Window w = window();
    const KeyWalk k = make_walk(a, b, w, T);
    for (int p : {a, b, (a + b) / 2}) {
      std::vector<int> shown(b + 1);
      const int reach = std::max(0, p - w.keys + 1);
      for (int i = 0; i < k.n; ++i) {
        const bool first = k.first_tokens(i);
        const int from = first ? 0 : reach, to = first ? std::min(w.sinks, reach) - 1 : p;
        const int read0 = first ? 0 : k.lo, read1 = (first ? k.first : k.end) - 1, t0 = k.tile(i) * T;
        CHECK(k.tile(i) >= 0 && t0 <= b && read0 <= read1);
        CHECK(i >= k.n_full || (!first && t0 >= read0 && t0 + T - 1 <= read1));
        for (int t = t0; t < t0 + T; ++t) {
          const bool sees = t >= from && t <= to;
          CHECK(sees || i >= k.n_full);
          if (!sees) continue;
          CHECK(t >= read0 && t <= read1);
          ++shown[t];
        }
      }
      for (int t = 0; t <= b; ++t)
        CHECK(shown[t] == (t <= p && (t > p - (int64_t)w.keys || t < w.sinks)));
    }
  }
  return 0;
}

// The ranges of a plan hold every visit of every row tile, at the ends of the positions' range too, and
// a plan keeps to the workspace that it is given.
static int plans() {
  const char* what = "plans";
  const int heads[][2] = {{1, 1}, {8, 1}, {8, 2}, {32, 8}, {12, 3}, {128, 2}};
  for (int it = 0; it < 4000; ++it) {
    const auto& hh = heads[upto(6)];
    const int gqa = hh[0] / hh[1], d = upto(2) ? 64 : 128;
    Window w = window();
    if (upto(3) == 0) w.keys = upto(2) ? 1 + upto(100000) : INT32_MAX;
    std::vector<SeqInput> seqs(1 + upto(upto(4) ? 4 : 90));
    int row = 0;
    for (auto& s : seqs) {
      const int chunk = upto(2) ? 1 : 1 + upto(900), prefix = upto(8) ? upto(30000) : INT32_MAX - chunk - upto(3);
      s = SeqInput{0, row, row, chunk, prefix};
      row += chunk;
    }
    const bool fp8 = upto(2);
    const Plan full = make_plan(seqs.data(), (int)seqs.size(), hh[0], hh[1], d, 256, SIZE_MAX, w, fp8);
    const size_t budget = full.min_bytes + (size_t)upto(1 << 20);
    const Plan tight = make_plan(seqs.data(), (int)seqs.size(), hh[0], hh[1], d, 256, budget, w, fp8);
    CHECK(tight.bytes <= std::max<size_t>(budget, 256));
    for (const Plan* plan : {&full, &tight}) {
      size_t n = 0;
      for (const LaunchPlan* lp : {&plan->rows, &plan->keys}) {
        n += lp->descs.size();
        for (const SeqDesc& sd : lp->descs) {
          const int64_t rows = (int64_t)sd.chunk_len * gqa;
          for (int64_t rt : {(int64_t)0, (int64_t)sd.n_row_tiles / 2, (int64_t)sd.n_row_tiles - 1}) {
            const int64_t r0 = rt * lp->shape.rows_per_wg, r1 = std::min(rows, r0 + lp->shape.rows_per_wg) - 1;
            const KeyWalk k = make_walk(sd.prefix_len + (int)(r0 / gqa), sd.prefix_len + (int)(r1 / gqa), w,
                                        lp->shape.tile_keys);
            CHECK(k.n >= 1 && k.n <= kv_tiles_of(sd, lp->shape));
            CHECK((int64_t)sd.n_split * sd.tiles_per_split >= k.n);
            // (blocks of a quarter of a key-split launch's tile)
            const KeyWalk q = make_walk(sd.prefix_len + (int)(r0 / gqa), sd.prefix_len + (int)(r1 / gqa), w, 32);
            CHECK(!lp->key_split || (int64_t)sd.n_split * sd.tiles_per_split * kWaves >= q.n);
          }
        }
      }
      CHECK(n == seqs.size());
    }
  }
  return 0;
}
int main() {
  if (walks() || plans()) return 1;
  std::printf("ok\n");
}
"""


def test_walks_and_plans(tmp_path):
    src, exe = tmp_path / "walks.hip", str(tmp_path / "walks")
    src.write_text(WALKS)
    res = subprocess.run([HIPCC, "-O1", *FLAGS, str(src), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "ok" in run.stdout, run.stdout + run.stderr


DRIVER = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "medha.h"
extern "C" const char no_kernels[4096] = {};
#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)
int main() {
  std::mt19937 rng(3);
  void* dev = (void*)0x100000;  // never read here
  for (int it = 0; it < 3000; ++it) {
    const int n = 1 + rng() % (it % 50 ? 8 : 3000);
    std::vector<int32_t> prefix(n), chunk(n);
    std::vector<int64_t> offs(n + 1);
    int64_t rows = 0;
    for (int i = 0; i < n; ++i) {
      chunk[i] = 1 + (rng() % 3 ? 0 : rng() % 4000);
      prefix[i] = rng() % 20 ? rng() % 100000 : INT32_MAX - chunk[i];
      offs[i + 1] = offs[i] + ((int64_t)prefix[i] + chunk[i] + 15) / 16;
      rows += chunk[i];
    }
    const int heads[][2] = {{1, 1}, {32, 8}, {128, 1}, {6, 3}};
    const auto& h = heads[rng() % 4];
    const int d = rng() % 2 ? 64 : 128, window = rng() % 3 ? 1 + rng() % 9000 : INT32_MAX, sinks = rng() % 2 ? rng() % 300 : INT32_MAX;
    const size_t a = medha_window_workspace_bytes(prefix.data(), chunk.data(), n, h[0], h[1], d, window, sinks);
    const size_t b = medha_chunked_prefill_fp8_workspace_bytes(prefix.data(), chunk.data(), n, h[0], h[1], d, window, sinks);
    CHECK(a >= 256 && b >= 256);
    CHECK(medha_chunked_prefill_fp8_workspace_bytes(prefix.data(), chunk.data(), n, h[0], h[1], d, 0, sinks) >= 256);
    // behind the planning: refused for scratch that is not there, or, where the rule needs none, ended by
    // the runtime, which has no device here
    medha_kv_cache kv{dev, dev, 10, 16, h[1], d};
    medha_kv_cache_fp8 k8{dev, dev, dev, 10, 16, h[1], d};
    if (a > (size_t)64 << 20) {
      const int rc = medha_window_attn(dev, &kv, (const int32_t*)dev, offs.data(), prefix.data(), chunk.data(), n, h[0], 1.f,
                                       window, sinks, 0, dev, (float*)dev, (char*)dev + 16, 1 << 20, nullptr);
      CHECK(rc == MEDHA_ERR_WORKSPACE || rc == MEDHA_ERR_HIP);
    }
    offs[n] = offs[n - 1];  // a slice too short is found before anything is enqueued
    CHECK(medha_window_attn(dev, &kv, (const int32_t*)dev, offs.data(), prefix.data(), chunk.data(), n, h[0], 1.f, window,
                            sinks, 1, dev, (float*)dev, dev, SIZE_MAX, nullptr) == MEDHA_ERR_INVALID_ARG);
    CHECK(medha_chunked_prefill_attn_fp8(dev, &k8, (const int32_t*)dev, offs.data(), prefix.data(), chunk.data(), n, h[0],
                                         1.f, window, sinks, 1, dev, (float*)dev, dev, SIZE_MAX, nullptr) ==
          MEDHA_ERR_INVALID_ARG);
    CHECK(medha_kv_append_fp8(dev, dev, &k8, (const int32_t*)dev, offs.data(), prefix.data(), chunk.data(), n, nullptr) ==
          MEDHA_ERR_INVALID_ARG);
    CHECK(medha_kv_read_fp8(&k8, (const int32_t*)dev, offs.data(), prefix.data(), chunk.data(), n, dev, dev, nullptr) ==
          MEDHA_ERR_INVALID_ARG);
  }
  std::printf("ok\n");
}
"""


def test_host_code_under_the_sanitizers(tmp_path):
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined"]
    src, lib, drv, exe = (str(tmp_path / n) for n in ("driver.cpp", "lib.o", "driver.o", "run"))
    open(src, "w").write(DRIVER)
    host_san = [x for f in san for x in ("-Xarch_host", f)]
    clang = "/opt/rocm/lib/llvm/bin/clang++"

    def build(*cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, " ".join(cmd) + "\n" + res.stderr[-4000:]
        return res.stdout

    # (the host's half alone, with nothing in the place of the kernels: none is launched)
    build(HIPCC, "-O1", "-g", *FLAGS, "--offload-host-only", *host_san, "-c",
          os.path.join(CSRC, "window_fp8.hip"), "-o", lib)
    build(clang, "-O1", "-g", "-std=c++17", *san, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", drv)
    names = [x.split()[-1] for x in build("nm", "-u", lib).splitlines()]
    stubs = [f"-Wl,--defsym,{x}=no_kernels" for x in names if x.startswith("__hip_fatbin")]
    build(HIPCC, "-fno-gpu-sanitize", *san, *stubs, lib, drv, "-o", exe)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1",
               HIP_VISIBLE_DEVICES="")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0 and "ok" in run.stdout, run.stdout[-2000:] + run.stderr[-6000:]
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr
