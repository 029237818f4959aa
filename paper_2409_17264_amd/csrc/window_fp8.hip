// C ABI of the 8-bit KV cache and of windowed attention: argument validation, launch planning and
// kernel launches.  See include/medha.h for the contract.
#include "medha.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.h"
#include "fp8_cache_kernel.h"
#include "host.h"
#include "planner.h"

namespace medha {
namespace {

int check_cache(const medha_kv_cache_fp8* kv) {
  if (kv == nullptr || kv->num_kv_heads <= 0 || kv->num_pages < 0) return MEDHA_ERR_INVALID_ARG;
  if (kv->page_size != kPageSize || (kv->head_dim != 64 && kv->head_dim != 128))
    return MEDHA_ERR_UNSUPPORTED;
  return MEDHA_OK;
}

// Both directions: tokens [first[b], first[b] + count[b]) of every sequence, `least` of them or more.
template <class Kernel>
int move_tokens(Kernel kernel, const void* k_rows, const void* v_rows, const medha_kv_cache_fp8* kv,
                const int32_t* page_table, const int64_t* page_table_offs, const int32_t* first,
                const int32_t* count, int32_t batch, int32_t least, void* hip_stream) {
  const int rc = check_cache(kv);
  if (rc != MEDHA_OK) return rc;
  if (batch < 0) return MEDHA_ERR_INVALID_ARG;
  if (batch == 0) return MEDHA_OK;
  if (k_rows == nullptr || v_rows == nullptr || kv->k_pool == nullptr || kv->v_pool == nullptr ||
      kv->scale == nullptr || page_table == nullptr || page_table_offs == nullptr ||
      first == nullptr || count == nullptr)
    return MEDHA_ERR_INVALID_ARG;
  if (!aligned(k_rows, 16) || !aligned(v_rows, 16) || !aligned(kv->k_pool, 16) ||
      !aligned(kv->v_pool, 16) || !aligned(kv->scale, 16) || !aligned(page_table, 4))
    return MEDHA_ERR_INVALID_ARG;
  int64_t rows = 0;
  for (int b = 0; b < batch; ++b) {
    if (first[b] < 0 || count[b] < least) return MEDHA_ERR_INVALID_ARG;
    if ((int64_t)first[b] + count[b] > INT32_MAX) return MEDHA_ERR_INVALID_ARG;
    const int64_t pages = ceil_div((int64_t)first[b] + count[b], kPageSize);
    if (page_table_offs[b] < 0 || page_table_offs[b + 1] - page_table_offs[b] < pages)
      return MEDHA_ERR_INVALID_ARG;
    rows += count[b];
    if (rows > INT32_MAX) return MEDHA_ERR_INVALID_ARG;
  }
  // validated in full before the first launch; up to kMaxInlineSeq sequences per launch
  int64_t src_row = 0;
  for (int b0 = 0; b0 < batch; b0 += kMaxInlineSeq) {
    Fp8CacheArgs a{};
    a.k_rows = static_cast<uint4*>(const_cast<void*>(k_rows));
    a.v_rows = static_cast<uint4*>(const_cast<void*>(v_rows));
    a.k_pool = static_cast<uint2*>(const_cast<void*>(kv->k_pool));
    a.v_pool = static_cast<uint2*>(const_cast<void*>(kv->v_pool));
    a.scale = static_cast<uint8_t*>(const_cast<void*>(kv->scale));
    a.page_table = page_table;
    a.h_kv = kv->num_kv_heads;
    a.words_per_row = kv->head_dim / 8;
    a.num_pages = kv->num_pages;
    a.n_seq = std::min(kMaxInlineSeq, batch - b0);
    int32_t rank = 0;
    for (int i = 0; i < a.n_seq; ++i) {
      a.descs[i] = AppendDesc{page_table_offs[b0 + i], (int32_t)src_row, first[b0 + i], count[b0 + i], rank};
      rank += count[b0 + i];
      src_row += count[b0 + i];
    }
    if (rank == 0) continue;
    a.total_rows = rank;
    const int64_t threads = (int64_t)rank * a.h_kv * a.words_per_row;
    const int64_t grid = std::min<int64_t>(ceil_div(threads, kThreads), 1 << 20);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), 0,
                       static_cast<hipStream_t>(hip_stream), a);
    if (hipGetLastError() != hipSuccess) return MEDHA_ERR_HIP;
  }
  return MEDHA_OK;
}

}  // namespace
}  // namespace medha

using namespace medha;

extern "C" {

int medha_kv_append_fp8(const void* k_new, const void* v_new, const medha_kv_cache_fp8* kv,
                        const int32_t* page_table, const int64_t* page_table_offs,
                        const int32_t* prefix_len, const int32_t* chunk_len, int32_t batch,
                        void* hip_stream) {
  return move_tokens(kv_append_fp8_kernel, k_new, v_new, kv, page_table, page_table_offs, prefix_len,
                     chunk_len, batch, 1, hip_stream);
}

int medha_kv_read_fp8(const medha_kv_cache_fp8* kv, const int32_t* page_table,
                      const int64_t* page_table_offs, const int32_t* first, const int32_t* count,
                      int32_t batch, void* k_out, void* v_out, void* hip_stream) {
  return move_tokens(kv_read_fp8_kernel, k_out, v_out, kv, page_table, page_table_offs, first, count,
                     batch, 0, hip_stream);
}

}  // extern "C"
