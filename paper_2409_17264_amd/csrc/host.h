// Host-side checks that the library's entry points share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "common.h"
#include "medha.h"

namespace medha {

inline int current_num_cus() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      cus <= 0) {
    (void)hipGetLastError();
    return 256;  // MI355X; used only for planning queries made without a device
  }
  return cus;
}

inline bool aligned(const void* p, size_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0;
}

inline int check_heads(int h_q, int h_kv, int d, int page_size) {
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0) return MEDHA_ERR_INVALID_ARG;
  if (page_size != kPageSize || (d != 64 && d != 128)) return MEDHA_ERR_UNSUPPORTED;
  return MEDHA_OK;
}

// The part of a caller's workspace a plan may count on: none of a missing or misaligned one.
inline size_t usable_bytes(const void* workspace, size_t bytes) {
  return workspace != nullptr && aligned(workspace, 256) ? bytes : 0;
}

}  // namespace medha
