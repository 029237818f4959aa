// C ABI of the 8-bit KV cache and of windowed attention: argument validation, launch planning and
// kernel launches.  See include/medha.h for the contract.
#include "medha.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <exception>
#include <vector>

#include "common.h"
#include "fp8_cache_kernel.h"
#include "host.h"
#include "medha_internal.h"
#include "merge_kernel.h"
#include "planner.h"
#include "walk_kernel.h"

namespace medha {
namespace {

int check_cache(const medha_kv_cache_fp8* kv) {
  if (kv == nullptr || kv->num_kv_heads <= 0 || kv->num_pages < 0) return MEDHA_ERR_INVALID_ARG;
  if (kv->page_size != kPageSize || (kv->head_dim != 64 && kv->head_dim != 128))
    return MEDHA_ERR_UNSUPPORTED;
  return MEDHA_OK;
}

// Both directions: tokens [first[b], first[b] + count[b]) of every sequence, `least` of them or more.
int move_tokens(bool append, const void* k_rows, const void* v_rows, const medha_kv_cache_fp8* kv,
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
  // K and V rows in bf16 (see kv_read_fp8_kernel)
  const bool once = rows * kv->num_kv_heads * kv->head_dim * 4 >= kLastLevelCacheBytes;
  const auto kernel = append ? kv_append_fp8_kernel
                      : once ? kv_read_fp8_kernel<true>
                             : kv_read_fp8_kernel<false>;
  // validated in full before the first launch; up to kMaxInlineSeq sequences per launch
  int64_t src_row = 0;
  for (int b0 = 0; b0 < batch; b0 += kMaxInlineSeq) {
    Fp8CacheArgs a{};
    a.k_rows = static_cast<uint4*>(const_cast<void*>(k_rows));
    a.v_rows = static_cast<uint4*>(const_cast<void*>(v_rows));
    a.k_pool = const_cast<void*>(kv->k_pool);
    a.v_pool = const_cast<void*>(kv->v_pool);
    a.scale = static_cast<uint8_t*>(const_cast<void*>(kv->scale));
    a.page_table = page_table;
    a.h_kv = kv->num_kv_heads;
    a.words_per_row = kv->head_dim / (append ? 16 : 8);
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

// ------------------------------------------------------------------ attention

// Over the bf16 cache a launch of more workgroups than compute units takes the small ring, so that two
// share one (64 decodes of 4K median behind a window of 4096, 32/8 heads, d 128, 141.8 -> 133.5 us; 128
// of 2K behind 1000 113.9 -> 103.6; 60 of 8K at 8/1 heads behind 300000 73.0 -> 66.9), one of fewer the
// large (8 of 2K behind 4096, 32/8 heads, 19.9 -> 17.9; 16 of 8K at 8/1 16.7 -> 15.6).
template <int D>
hipError_t launch_keys(const LaunchPlan& lp, const WalkArgs& a, int grid, hipStream_t stream) {
  if (a.scale != nullptr)
    hipLaunchKernelGGL((key_walk_kernel<D, Fp8Block<D>, 2>), dim3(grid), dim3(kThreads), 0, stream, a);
  else if (grid > lp.num_cus)
    hipLaunchKernelGGL((key_walk_kernel<D, Bf16Block<D>, 1>), dim3(grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((key_walk_kernel<D, Bf16Block<D>, 2>), dim3(grid), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <int D, bool kFp8>
hipError_t launch_rows(const LaunchPlan& lp, const WalkArgs& a, int grid, hipStream_t stream) {
  if (lp.q_blocks == 2)
    hipLaunchKernelGGL((row_walk_kernel<D, 8, kFp8>), dim3(grid), dim3(512), 0, stream, a);
  else if (lp.paired)
    hipLaunchKernelGGL((row_walk_kernel<128, 4, kFp8, true>), dim3(grid), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((row_walk_kernel<D, 4, kFp8>), dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <int D, class Out>
hipError_t launch_merge(const MergeArgs& m, int max_split, hipStream_t stream) {
  if (max_split > kWideMergeSplits) {
    const int64_t blocks = (int64_t)m.total_rows * m.h_q;
    hipLaunchKernelGGL((split_merge_wide_kernel<D, Out, true>), dim3((unsigned)blocks),
                       dim3(kThreads), 0, stream, m);
  } else {
    const int64_t threads = (int64_t)m.total_rows * m.h_q * (D / 4);
    hipLaunchKernelGGL((split_merge_kernel<D, Out, true>), dim3((unsigned)ceil_div(threads, kThreads)),
                       dim3(kThreads), 0, stream, m);
  }
  return hipGetLastError();
}

// Launches one mode's sequences, at most kMaxInlineSeq per kernel launch, each followed by the
// merge of its split-KV partials.
template <int D>
hipError_t launch_walks(const LaunchPlan& lp, WalkArgs& a, hipStream_t stream) {
  if (lp.descs.empty() || lp.n_slots == 0) return hipSuccess;
  const int n_all = (int)lp.descs.size();
  for (int g0 = 0; g0 < n_all; g0 += kMaxInlineSeq) {
    const int n = std::min(kMaxInlineSeq, n_all - g0);
    const int slot0 = lp.descs[g0].work_start, rank0 = lp.descs[g0].row_rank;
    const int slot1 = g0 + n < n_all ? lp.descs[g0 + n].work_start : lp.n_slots;
    const int rank1 = g0 + n < n_all ? lp.descs[g0 + n].row_rank : lp.total_rows;
    a.n_seq = n;
    int max_split = 1;
    for (int i = 0; i < n; ++i) {
      SeqDesc& sd = a.inline_descs[i];
      sd = lp.descs[g0 + i];
      sd.work_start -= slot0;
      sd.row_rank -= rank0;
      max_split = std::max(max_split, sd.n_split);
    }
    if (slot1 == slot0) continue;
    hipError_t e = lp.key_split         ? launch_keys<D>(lp, a, slot1 - slot0, stream)
                   : a.scale != nullptr ? launch_rows<D, true>(lp, a, slot1 - slot0, stream)
                                        : launch_rows<D, false>(lp, a, slot1 - slot0, stream);
    if (e != hipSuccess) return e;
    if (max_split == 1) continue;
    MergeArgs m{};
    m.part_o = a.part_o;
    m.part_lse = a.part_lse;
    m.out = static_cast<float*>(a.out);
    m.lse = a.lse;
    m.n_seq = n;
    m.h_q = a.h_q;
    m.total_rows = rank1 - rank0;
    std::memcpy(m.inline_descs, a.inline_descs, n * sizeof(SeqDesc));
    e = a.out_bf16 ? launch_merge<D, __bf16>(m, max_split, stream)
                   : launch_merge<D, float>(m, max_split, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The window of a call: 0 keys mean none, where that is allowed.
bool window_of(int32_t keys, int32_t sinks, bool optional, Window& w) {
  w = Window{};
  if (optional && keys == 0) return true;
  if (keys < 1 || sinks < 0) return false;
  w.keys = keys;
  w.sinks = sinks;
  return true;
}

Plan walk_plan(const std::vector<SeqInput>& seqs, int h_q, int h_kv, int d, size_t budget,
               const Window& w, bool fp8) {
  return make_plan(seqs.data(), (int)seqs.size(), h_q, h_kv, d, current_num_cus(), budget, w, fp8);
}

size_t walk_workspace(const int32_t* prefix_len, const int32_t* chunk_len, int32_t batch,
                      int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t window,
                      int32_t sinks, bool fp8) {
  Window w;
  if (batch < 0 || (batch > 0 && (prefix_len == nullptr || chunk_len == nullptr))) return 0;
  if (check_heads(num_q_heads, num_kv_heads, head_dim, kPageSize) != MEDHA_OK) return 0;
  if (!window_of(window, sinks, fp8, w)) return 0;
  std::vector<SeqInput> seqs(batch);
  int64_t row = 0;
  for (int b = 0; b < batch; ++b) {
    if (prefix_len[b] < 0 || chunk_len[b] < 1) return 0;
    if ((int64_t)prefix_len[b] + chunk_len[b] > INT32_MAX) return 0;
    seqs[b] = SeqInput{0, (int32_t)row, (int32_t)row, chunk_len[b], prefix_len[b]};
    row += chunk_len[b];
    if (row > INT32_MAX) return 0;
  }
  return walk_plan(seqs, num_q_heads, num_kv_heads, head_dim, SIZE_MAX, w, fp8)
      .workspace_bytes();
}

// A call on either cache.  `kv` describes its pools, `scale` is null for the bf16 one; `alloc`: asked
// for a workspace of the reported size instead of the caller's.
int walk_attn(const void* q, const medha_kv_cache* kv, const void* scale, const int32_t* page_table,
              const int64_t* page_table_offs, const int32_t* prefix_len, const int32_t* chunk_len,
              int32_t batch, int32_t num_q_heads, float softmax_scale, const Window& window,
              int32_t out_type, void* out, float* lse, void* workspace, size_t workspace_bytes,
              medha_alloc alloc, void* context, void* hip_stream) {
  if (batch < 0) return MEDHA_ERR_INVALID_ARG;
  if (kv->k_pool == nullptr || kv->v_pool == nullptr || kv->num_pages <= 0)
    return MEDHA_ERR_INVALID_ARG;
  if (!aligned(kv->k_pool, 16) || !aligned(kv->v_pool, 16) || !aligned(scale, 16))
    return MEDHA_ERR_INVALID_ARG;
  const int rc = check_heads(num_q_heads, kv->num_kv_heads, kv->head_dim, kv->page_size);
  if (rc != MEDHA_OK) return rc;
  if (out_type != MEDHA_OUT_FP32 && out_type != MEDHA_OUT_BF16) return MEDHA_ERR_INVALID_ARG;
  if (batch == 0) return MEDHA_OK;
  if (q == nullptr || page_table == nullptr || page_table_offs == nullptr ||
      prefix_len == nullptr || chunk_len == nullptr || out == nullptr || lse == nullptr)
    return MEDHA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(page_table, 4) ||
      !std::isfinite(softmax_scale))
    return MEDHA_ERR_INVALID_ARG;
  std::vector<SeqInput> seqs(batch);
  int64_t row = 0;
  for (int b = 0; b < batch; ++b) {
    if (prefix_len[b] < 0 || chunk_len[b] < 1) return MEDHA_ERR_INVALID_ARG;
    const int64_t n = (int64_t)prefix_len[b] + chunk_len[b];
    if (n > INT32_MAX) return MEDHA_ERR_INVALID_ARG;
    const int64_t have = page_table_offs[b + 1] - page_table_offs[b];
    if (page_table_offs[b] < 0 || have < ceil_div(n, kPageSize)) return MEDHA_ERR_INVALID_ARG;
    seqs[b] = SeqInput{page_table_offs[b], (int32_t)row, (int32_t)row, chunk_len[b], prefix_len[b]};
    row += chunk_len[b];
    if (row > INT32_MAX) return MEDHA_ERR_INVALID_ARG;
  }
  const Plan plan = walk_plan(seqs, num_q_heads, kv->num_kv_heads, kv->head_dim,
                              alloc ? SIZE_MAX : usable_bytes(workspace, workspace_bytes), window,
                              scale != nullptr);
  if (alloc) {
    workspace_bytes = plan.workspace_bytes();
    workspace = alloc(workspace_bytes, context);
    if (workspace == nullptr) return MEDHA_ERR_WORKSPACE;
  }
  if (plan.part_rows > 0 || plan.min_part_rows > 0) {
    if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < plan.min_bytes ||
        workspace_bytes < plan.bytes)
      return MEDHA_ERR_WORKSPACE;
  }
  char* ws = static_cast<char*>(workspace);
  WalkArgs a{};
  a.q = static_cast<const __bf16*>(q);
  a.k_pool = static_cast<const char*>(kv->k_pool);
  a.v_pool = static_cast<const char*>(kv->v_pool);
  a.scale = static_cast<const uint8_t*>(scale);
  a.page_table = page_table;
  a.out = out;
  a.lse = lse;
  a.part_o = ws ? reinterpret_cast<float*>(ws + plan.off_part_o) : nullptr;
  a.part_lse = ws ? reinterpret_cast<float*>(ws + plan.off_part_lse) : nullptr;
  a.h_q = num_q_heads;
  a.h_kv = kv->num_kv_heads;
  a.scale_log2 = softmax_scale * kLog2e;
  a.window = window;
  a.out_bf16 = out_type == MEDHA_OUT_BF16;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const auto launch = kv->head_dim == 128 ? launch_walks<128> : launch_walks<64>;
  if (launch(plan.rows, a, stream) != hipSuccess || launch(plan.keys, a, stream) != hipSuccess)
    return MEDHA_ERR_HIP;
  return MEDHA_OK;
}

int attn_bf16(const void* q, const medha_kv_cache* kv, const int32_t* page_table,
              const int64_t* page_table_offs, const int32_t* prefix_len, const int32_t* chunk_len,
              int32_t batch, int32_t num_q_heads, float softmax_scale, int32_t window,
              int32_t sinks, int32_t out_type, void* out, float* lse, void* workspace,
              size_t workspace_bytes, medha_alloc alloc, void* context, void* hip_stream) {
  Window w;
  if (kv == nullptr || !window_of(window, sinks, false, w)) return MEDHA_ERR_INVALID_ARG;
  return walk_attn(q, kv, nullptr, page_table, page_table_offs, prefix_len, chunk_len, batch,
                   num_q_heads, softmax_scale, w, out_type, out, lse, workspace, workspace_bytes,
                   alloc, context, hip_stream);
}

int attn_fp8(const void* q, const medha_kv_cache_fp8* kv, const int32_t* page_table,
             const int64_t* page_table_offs, const int32_t* prefix_len, const int32_t* chunk_len,
             int32_t batch, int32_t num_q_heads, float softmax_scale, int32_t window, int32_t sinks,
             int32_t out_type, void* out, float* lse, void* workspace, size_t workspace_bytes,
             medha_alloc alloc, void* context, void* hip_stream) {
  Window w;
  if (kv == nullptr || kv->scale == nullptr || !window_of(window, sinks, true, w))
    return MEDHA_ERR_INVALID_ARG;
  const medha_kv_cache pools{kv->k_pool, kv->v_pool, kv->num_pages, kv->page_size,
                             kv->num_kv_heads, kv->head_dim};
  return walk_attn(q, &pools, kv->scale, page_table, page_table_offs, prefix_len, chunk_len, batch,
                   num_q_heads, softmax_scale, w, out_type, out, lse, workspace, workspace_bytes,
                   alloc, context, hip_stream);
}

// Runs a call whose host memory may not be there: no exception leaves the library.
template <class F>
auto guarded(F&& call, decltype(call()) refused) -> decltype(call()) {
  try {
    return call();
  } catch (const std::exception&) {
    return refused;
  }
}

}  // namespace
}  // namespace medha

using namespace medha;

extern "C" {

int medha_kv_append_fp8(const void* k_new, const void* v_new, const medha_kv_cache_fp8* kv,
                        const int32_t* page_table, const int64_t* page_table_offs,
                        const int32_t* prefix_len, const int32_t* chunk_len, int32_t batch,
                        void* hip_stream) {
  return move_tokens(true, k_new, v_new, kv, page_table, page_table_offs, prefix_len,
                     chunk_len, batch, 1, hip_stream);
}

int medha_kv_read_fp8(const medha_kv_cache_fp8* kv, const int32_t* page_table,
                      const int64_t* page_table_offs, const int32_t* first, const int32_t* count,
                      int32_t batch, void* k_out, void* v_out, void* hip_stream) {
  return move_tokens(false, k_out, v_out, kv, page_table, page_table_offs, first, count,
                     batch, 0, hip_stream);
}

size_t medha_window_workspace_bytes(const int32_t* prefix_len, const int32_t* chunk_len,
                                    int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                    int32_t head_dim, int32_t window, int32_t sinks) {
  return guarded([&] {
    return walk_workspace(prefix_len, chunk_len, batch, num_q_heads, num_kv_heads, head_dim, window,
                          sinks, false);
  }, (size_t)0);
}

int medha_window_attn(const void* q, const medha_kv_cache* kv, const int32_t* page_table,
                      const int64_t* page_table_offs, const int32_t* prefix_len,
                      const int32_t* chunk_len, int32_t batch, int32_t num_q_heads,
                      float softmax_scale, int32_t window, int32_t sinks, int32_t out_type,
                      void* out, float* lse, void* workspace, size_t workspace_bytes,
                      void* hip_stream) {
  return guarded([&] {
    return attn_bf16(q, kv, page_table, page_table_offs, prefix_len, chunk_len, batch, num_q_heads,
                     softmax_scale, window, sinks, out_type, out, lse, workspace, workspace_bytes,
                     nullptr, nullptr, hip_stream);
  }, MEDHA_ERR_MEMORY);
}

int medha_window_attn_alloc(const void* q, const medha_kv_cache* kv, const int32_t* page_table,
                            const int64_t* page_table_offs, const int32_t* prefix_len,
                            const int32_t* chunk_len, int32_t batch, int32_t num_q_heads,
                            float softmax_scale, int32_t window, int32_t sinks, int32_t out_type,
                            void* out, float* lse, medha_alloc alloc, void* context,
                            void* hip_stream) {
  if (alloc == nullptr) return MEDHA_ERR_INVALID_ARG;
  return guarded([&] {
    return attn_bf16(q, kv, page_table, page_table_offs, prefix_len, chunk_len, batch, num_q_heads,
                     softmax_scale, window, sinks, out_type, out, lse, nullptr, 0, alloc, context,
                     hip_stream);
  }, MEDHA_ERR_MEMORY);
}

size_t medha_chunked_prefill_fp8_workspace_bytes(const int32_t* prefix_len,
                                                 const int32_t* chunk_len, int32_t batch,
                                                 int32_t num_q_heads, int32_t num_kv_heads,
                                                 int32_t head_dim, int32_t window, int32_t sinks) {
  return guarded([&] {
    return walk_workspace(prefix_len, chunk_len, batch, num_q_heads, num_kv_heads, head_dim, window,
                          sinks, true);
  }, (size_t)0);
}

int medha_chunked_prefill_attn_fp8(const void* q, const medha_kv_cache_fp8* kv,
                                   const int32_t* page_table, const int64_t* page_table_offs,
                                   const int32_t* prefix_len, const int32_t* chunk_len,
                                   int32_t batch, int32_t num_q_heads, float softmax_scale,
                                   int32_t window, int32_t sinks, int32_t out_type, void* out,
                                   float* lse, void* workspace, size_t workspace_bytes,
                                   void* hip_stream) {
  return guarded([&] {
    return attn_fp8(q, kv, page_table, page_table_offs, prefix_len, chunk_len, batch, num_q_heads,
                    softmax_scale, window, sinks, out_type, out, lse, workspace, workspace_bytes,
                    nullptr, nullptr, hip_stream);
  }, MEDHA_ERR_MEMORY);
}

int medha_chunked_prefill_attn_fp8_alloc(const void* q, const medha_kv_cache_fp8* kv,
                                         const int32_t* page_table, const int64_t* page_table_offs,
                                         const int32_t* prefix_len, const int32_t* chunk_len,
                                         int32_t batch, int32_t num_q_heads, float softmax_scale,
                                         int32_t window, int32_t sinks, int32_t out_type, void* out,
                                         float* lse, medha_alloc alloc, void* context,
                                         void* hip_stream) {
  if (alloc == nullptr) return MEDHA_ERR_INVALID_ARG;
  return guarded([&] {
    return attn_fp8(q, kv, page_table, page_table_offs, prefix_len, chunk_len, batch, num_q_heads,
                    softmax_scale, window, sinks, out_type, out, lse, nullptr, 0, alloc, context,
                    hip_stream);
  }, MEDHA_ERR_MEMORY);
}

}  // extern "C"
