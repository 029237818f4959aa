"""Windowed attention and the 8-bit cache when host memory runs out (CPU): the host code of their entry points
with an allocator that refuses."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CSRC = os.path.join(ROOT, "paper_2409_17264_amd", "csrc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")

DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "medha.h"
#include "medha_internal.h"
extern "C" const char no_kernels[4096] = {};
static long left = -1;  // allocations that still succeed; all of them below 0
void* operator new(std::size_t n) {
  if (left == 0) throw std::bad_alloc();
  if (left > 0) --left;
  return std::malloc(n ? n : 1);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)
static void* none(size_t, void*) { return nullptr; }
int main() {
  const int32_t prefix[] = {30000, 5, 700}, chunk[] = {1, 300, 40};
  const int64_t offs[] = {0, 2000, 2100, 2200};
  void* dev = (void*)0x100000;  // never read here
  medha_kv_cache kv{dev, dev, 10, 16, 2, 128};
  medha_kv_cache_fp8 k8{dev, dev, dev, 10, 16, 2, 128};
  for (int call = 0; call < 6; ++call) {
    auto run = [&]() -> long {
      const int32_t* t = (const int32_t*)dev;
      float* f = (float*)dev;
      switch (call) {
        case 0: return medha_window_attn(dev, &kv, t, offs, prefix, chunk, 3, 8, 1.f, 9000, 4, 0, dev, f, dev, 256, nullptr);
        case 1: return medha_window_attn_alloc(dev, &kv, t, offs, prefix, chunk, 3, 8, 1.f, 9000, 4, 0, dev, f, none, nullptr, nullptr);
        case 2: return medha_chunked_prefill_attn_fp8(dev, &k8, t, offs, prefix, chunk, 3, 8, 1.f, 0, 0, 1, dev, f, dev, 256, nullptr);
        case 3: return medha_chunked_prefill_attn_fp8_alloc(dev, &k8, t, offs, prefix, chunk, 3, 8, 1.f, 0, 0, 1, dev, f, none, nullptr, nullptr);
        case 4: return (long)medha_window_workspace_bytes(prefix, chunk, 3, 8, 2, 128, 9000, 4);
        default: return (long)medha_chunked_prefill_fp8_workspace_bytes(prefix, chunk, 3, 8, 2, 128, 0, 0);
      }
    };
    const long with_memory = run();
    CHECK(call < 4 ? with_memory == MEDHA_ERR_WORKSPACE : with_memory > 256);
    int refused = 0;
    for (long n = 0; n < 100000; ++n) {
      left = n;
      const long got = run();
      const bool ran_out = left == 0;
      left = -1;
      if (got == with_memory) {
        CHECK(n > 0 && refused > 0);
        break;
      }
      CHECK(ran_out && got == (call < 4 ? MEDHA_ERR_MEMORY : 0));
      ++refused;
    }
  }
  std::printf("ok\n");
}
"""


def test_a_plan_without_host_memory(tmp_path):
    src, lib, drv, exe = (str(tmp_path / n) for n in ("driver.cpp", "lib.o", "driver.o", "run"))
    open(src, "w").write(DRIVER)

    def build(*cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, " ".join(cmd) + "\n" + res.stderr[-4000:]
        return res.stdout

    build(HIPCC, "-O1", "-g", "--offload-arch=gfx950", "-std=c++17", "-Wno-inline-asm", "-I", CSRC, "-I",
          os.path.join(ROOT, "include"), "--offload-host-only", "-c", os.path.join(CSRC, "window_fp8.hip"), "-o", lib)
    build("/opt/rocm/lib/llvm/bin/clang++", "-O1", "-g", "-std=c++17", "-I", CSRC, "-I",
          os.path.join(ROOT, "include"), "-c", src, "-o", drv)
    names = [x.split()[-1] for x in build("nm", "-u", lib).splitlines()]
    stubs = [f"-Wl,--defsym,{x}=no_kernels" for x in names if x.startswith("__hip_fatbin")]
    build(HIPCC, *stubs, lib, drv, "-o", exe)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120,
                         env=dict(os.environ, HIP_VISIBLE_DEVICES=""))
    assert run.returncode == 0 and "ok" in run.stdout, run.stdout[-2000:] + run.stderr[-3000:]
