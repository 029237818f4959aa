// Attention over a paged cache in 8 bits, and behind a sliding window over either cache.
//
//   O[r] = sum_t p[r,t] V[t] / l[r],  p[r,t] = exp(scale * q[r].K[t] - m[r]),  l[r] = sum_t p[r,t],
//   LSE[r] = m[r] + ln l[r],  t over the keys that row r sees,
//
// in one pass with a running maximum m and sum l (fp32).  Two ways to share the work out:
//   key_walk_kernel  32 query rows or fewer (decodes): they are read against few rows, so the bytes of
//                    the cache bound it; the walk is cut into ranges for the whole device to stream.
//   row_walk_kernel  chunks: 128 or 256 rows against each tile of 64 keys, so the matrix cores and the
//                    softmax's instructions beside them bound it, not memory.
// The keys that the rows of a workgroup see come as a KeyWalk.  Only keys that some row of the
// workgroup sees are read: the pages between the first tokens and the windows may be gone.
#pragma once

#include <type_traits>

#include "common.h"
#include "decode_kernel.h"
#include "fp8_cache_kernel.h"
#include "merge_kernel.h"
#include "prefill_kernel.h"
#include "walk.h"

namespace medha {

typedef int i32x2 __attribute__((ext_vector_type(2)));

struct WalkArgs {
  const __bf16* q;
  const char* k_pool;
  const char* v_pool;
  const uint8_t* scale;  // 8-bit cache only
  const int32_t* page_table;
  void* out;             // fp32, or bf16 if out_bf16
  float* lse;
  float* part_o;
  float* part_lse;
  int32_t n_seq;
  int32_t h_q;
  int32_t h_kv;
  float scale_log2;
  Window window;
  int32_t out_bf16;
  int32_t reserved;
  SeqDesc inline_descs[kMaxInlineSeq];
};
static_assert(sizeof(WalkArgs) <= 4096, "kernel argument block too large");

// What a row sees in a visit: the keys of one interval.  A lane's 32 keys of a 64-key tile (16 of a
// 32-key block) ascend with its registers -- key 8 (f / 4) + 4 half + f % 4 in register f -- so the
// interval is a run of bits, made once a visit, and masking takes two instructions a score: a bit
// spread over a register, and a selection by it.  (With two comparisons of the key against the
// interval's ends, four: eight prompts at d 64, window 1000, 149.5 -> 145 us; 64 decodes, window 4096,
// 163.7 -> 161.4.)
struct WindowMask {
  int position;   // of the row
  Window window;  // (wave-uniform)
  uint32_t bits;  // of the visit
  __device__ __forceinline__ float shown(float s, int, int f) const {
    const int all = (int)(bits << (31 - f)) >> 31;
    return __builtin_bit_cast(float, (all & __builtin_bit_cast(int, s)) | (~all & (int)0xff800000));
  }
  __device__ __forceinline__ void visit(bool first_tokens, int key0, int half) {
    const int reach = max(0, position - window.keys + 1);
    const int from = first_tokens ? 0 : reach;
    const int to = first_tokens ? min(window.sinks, reach) - 1 : position;
    bits = below(to + 1 - key0 - 4 * half) & ~below(from - key0 - 4 * half);
  }

 private:
  // the registers whose keys lie below x, counted from the lane's first
  static __device__ __forceinline__ uint32_t below(int x) {
    x = min(max(x, 0), 64);
    const int n = (x >> 3) * 4 + min(x & 7, 4);
    return (uint32_t)((1ull << n) - 1);
  }
};

// Where the keys of a visit are read from: keys that no row sees in it stand for the nearest one that
// some row does (they are masked, but have to be finite, and their pages may be gone).
struct KeyRange {
  int from, to;
  __device__ __forceinline__ KeyRange(const KeyWalk& w, bool first_tokens)
      : from(first_tokens ? 0 : w.lo), to((first_tokens ? w.first : w.end) - 1) {}
  __device__ __forceinline__ int key(int t) const { return min(max(t, from), to); }
  // the page, in the sequence's table, of the 16 keys from t on (a multiple of 16)
  __device__ __forceinline__ int page_index(int t) const { return key(t) >> 4; }
};

__device__ __forceinline__ void async_load4(const void* base_uniform, uint32_t lane_off,
                                            uint32_t lds_addr_uniform) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds_addr_uniform), "v"(lane_off), "s"(base_uniform)
               : "m0", "memory");
}

__device__ __forceinline__ void async_load4_at(const void* gptr, uint32_t lds_addr_uniform) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(lds_addr_uniform), "v"(gptr)
               : "m0", "memory");
}

// ---------------------------------------------------------------- blocks of 32 keys, bf16 cache

template <int D>
struct Bf16Block {
  using G = DecodeGeom<D>;
  using Rows = RowBlock<D, WindowMask>;
  static constexpr int kBytes = G::kBlockBytes;  // ring stage: K, V
  static constexpr int kLoads = G::kLoadsPerBlock;
  static constexpr int kPerPage = kPageSize / G::kRowsPerInstr;
  uint32_t k_off[kPerPage], v_off[kPerPage];  // of a whole page, within the (page, KV head) block
  int r_in, pos, half;

  __device__ __forceinline__ void init(int lane) {
    r_in = lane / G::kChunksPerRow;
    pos = lane % G::kChunksPerRow;
    half = lane >> 5;
#pragma unroll
    for (int j = 0; j < kPerPage; ++j) {
      const int r = j * G::kRowsPerInstr + r_in;
      k_off[j] = r * (D * 2) + Swz<D>::k(r, pos) * 16;
      v_off[j] = r * (D * 2) + Swz<D>::v(r, pos) * 16;
    }
  }

  __device__ static __forceinline__ void load_q(Rows& rb, const WalkArgs& args, const __bf16* qp,
                                                bool valid, int half) {
    const unsigned flip = args.scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int sl = 0; sl < Rows::kSlices; ++sl) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (valid) raw = *reinterpret_cast<const uint4*>(qp + sl * 16 + half * 8);
      raw.x ^= flip; raw.y ^= flip; raw.z ^= flip; raw.w ^= flip;
      rb.q[sl] = __builtin_bit_cast(bf16x8, raw);
    }
  }

  // Loads the block at key0 into `stage`; the ids of its two pages are page[0] and page[1].  WHOLE: all
  // of its keys are read.
  template <bool WHOLE, bool kOnce>
  __device__ __forceinline__ void issue(const WalkArgs& args, const int (&page)[2], const KeyRange& range,
                                        int key0, int kv_head, uint32_t stage) const {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int64_t block = ((int64_t)page[p] * args.h_kv + kv_head) * (kPageSize * D * 2);
      const char *kp = args.k_pool + block, *vp = args.v_pool + block;
#pragma unroll
      for (int j = 0; j < kPerPage; ++j) {
        uint32_t ko = k_off[j], vo = v_off[j];
        if (!WHOLE) {
          const int r = j * G::kRowsPerInstr + r_in, slot = range.key(key0 + p * kPageSize + r) & 15;
          ko = slot * (D * 2) + Swz<D>::k(r, pos) * 16;
          vo = slot * (D * 2) + Swz<D>::v(r, pos) * 16;
        }
        const uint32_t to = stage + (p * kPageSize + j * G::kRowsPerInstr) * (D * 2);
        async_load16<kOnce>(kp, ko, to);
        async_load16<kOnce>(vp, vo, to + G::kHalfBytes);
      }
    }
  }

  template <bool MASK>
  __device__ __forceinline__ void step(Rows& rb, const char* stage, int key0) const {
    rb.template step<1, MASK>(stage, stage + G::kHalfBytes, key0, half);
  }
};

// ---------------------------------------------------------------- a block of 32 keys, 8-bit cache

// 16-byte chunk of a row of D bytes, so that 16 rows read at one logical chunk hit all banks.
template <int D>
__device__ __forceinline__ int swz8(int row, int chunk) {
  return D == 128 ? (chunk ^ ((row >> 1) & 7)) : (chunk ^ ((row >> 2) & 3));
}

template <int D>
struct Fp8Block {
  using Rows = RowBlock<D, WindowMask>;
  static constexpr int kParts = D / 64;
  static constexpr int kHalfBytes = 32 * D;
  static constexpr int kBytes = 2 * kHalfBytes + 256;   // K, V, and 64 lanes' worth of scale bytes
  static constexpr int kChunksPerRow = D / 16;
  static constexpr int kRowsPerInstr = 64 / kChunksPerRow;  // 8 or 16
  static constexpr int kPerPage = kPageSize / kRowsPerInstr;
  static constexpr int kLoads = 4 * kPerPage + 1;
  uint32_t k_off[kPerPage], v_off[kPerPage];
  int k8_off[2 * kParts];          // this lane's pieces of key row lane % 32
  int vt_off[Rows::kDBlocks];      // its place in the transposing reads of a 16-key slice
  int ks_off, r_in, pos, lane, half;

  // 16-byte chunk of a V row: the 8 rows x 32 columns that 32 lanes read at a time hit all banks.
  __device__ static __forceinline__ int vswz(int row, int chunk) {
    const int g = D == 128 ? ((row >> 1) & 1) * 2 + ((row >> 3) & 1) * 4 : ((row >> 3) & 1) * 2;
    return chunk ^ g;
  }

  __device__ __forceinline__ void init(int ln) {
    lane = ln;
    half = ln >> 5;
    r_in = ln / kChunksPerRow;
    pos = ln % kChunksPerRow;
#pragma unroll
    for (int j = 0; j < kPerPage; ++j) {
      const int r = j * kRowsPerInstr + r_in;
      k_off[j] = r * D + swz8<D>(r, pos) * 16;
      v_off[j] = r * D + vswz(r, pos) * 16;
    }
    const int col = ln & 31;
#pragma unroll
    for (int i = 0; i < 2 * kParts; ++i)
      k8_off[i] = col * D + swz8<D>(col, (i >> 1) * 4 + half * 2 + (i & 1)) * 16;
    ks_off = (col >> 4) * kScaleBytesPerPage + (col & 15);
    // keys of a slice in the order of P^T's registers: 4*half + 0..3, then the same + 8
    const int l16 = ln & 15, dhalf = (ln >> 4) & 1, j = l16 >> 1;
    const int row = (j & 4) * 2 + 4 * half + (j & 3);
#pragma unroll
    for (int db = 0; db < Rows::kDBlocks; ++db)
      vt_off[db] = row * D + vswz(row, 2 * db + dhalf) * 16 + (l16 & 1) * 8;
  }

  // This half's elements of a query row are 32 of every 64, in the order of the keys' pieces.
  __device__ static __forceinline__ void load_q(Rows& rb, const WalkArgs& args, const __bf16* qp,
                                                bool valid, int half) {
    const unsigned flip = args.scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (valid) raw = *reinterpret_cast<const uint4*>(qp + (i / 4) * 64 + half * 32 + (i % 4) * 8);
      raw.x ^= flip; raw.y ^= flip; raw.z ^= flip; raw.w ^= flip;
      rb.q[i] = __builtin_bit_cast(bf16x8, raw);
    }
  }

  template <bool WHOLE, bool kOnce>
  __device__ __forceinline__ void issue(const WalkArgs& args, const int (&page)[2], const KeyRange& range,
                                        int key0, int kv_head, uint32_t stage) const {
    int64_t block[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      block[p] = (int64_t)page[p] * args.h_kv + kv_head;
      const char* kp = args.k_pool + block[p] * (kPageSize * D);
      const char* vp = args.v_pool + block[p] * (kPageSize * D);
#pragma unroll
      for (int j = 0; j < kPerPage; ++j) {
        uint32_t ko = k_off[j], vo = v_off[j];
        if (!WHOLE) {
          const int r = j * kRowsPerInstr + r_in, slot = range.key(key0 + p * kPageSize + r) & 15;
          ko = slot * D + swz8<D>(r, pos) * 16;
          vo = slot * D + vswz(r, pos) * 16;
        }
        const uint32_t to = stage + (p * kPageSize + j * kRowsPerInstr) * D;
        async_load16<kOnce>(kp, ko, to);
        async_load16<kOnce>(vp, vo, to + kHalfBytes);
      }
    }
    // (lanes 0-7 and 8-15 hold the two pages' 32 bytes, the others repeat them)
    const int64_t b = (lane & 8) ? block[1] : block[0];
    async_load4_at(args.scale + b * kScaleBytesPerPage + (lane & 7) * 4, stage + 2 * kHalfBytes);
  }

  // A lane turns its pieces of a key into bf16, scale and all: exact, and the sums are fp32 (an LSE over
  // 64 keys is off by 2e-7).
  // The values stay 8 bits wide until the transposing reads have them in registers.  There they
  // become bf16 without their scales, which differ from key to key: the scale of key t is a factor of
  // P[t] instead, a power of two, so nothing is rounded that would not have been: the values, up to 2^8,
  // give P 7 powers of two from their own range, which puts the scales, 2^-117 to 2^120, at 2^-110 to
  // 2^127, and a probability keeps bf16's 8 bits down to 2^-16 of its row's largest at the least of them.
  template <bool MASK>
  __device__ __forceinline__ void step(Rows& rb, const char* stage, int key0) const {
    const char* scales = stage + 2 * kHalfBytes;
    const char* v_lds = stage + kHalfBytes;
    i32x2 raw[2][Rows::kDBlocks];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int db = 0; db < Rows::kDBlocks; ++db)
        raw[g][db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (i32x2 __attribute__((address_space(3)))*)(v_lds + g * 16 * D + vt_off[db]));
    uint32_t vs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      vs[i] = *reinterpret_cast<const uint32_t*>(scales + (i >> 1) * kScaleBytesPerPage + kPageSize +
                                                 (i & 1) * 8 + half * 4);
    const float ks = scale_of((uint8_t)scales[ks_off]);
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * kParts; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(stage + k8_off[i]);
      const bf16x8 a = __builtin_bit_cast(bf16x8, dequantise8(make_uint2(x.x, x.y), ks));
      const bf16x8 b = __builtin_bit_cast(bf16x8, dequantise8(make_uint2(x.z, x.w), ks));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, rb.q[2 * i], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, rb.q[2 * i + 1], s, 0, 0, 0);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (MASK) s[e] = rb.mask.shown(s[e], 0, e);
      mx = fmaxf(mx, s[e]);
    }
    const float m_use = rb.template update_reference<MASK>(mx);
    float ls = 0.f;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      f32x8 pe;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float pr = rb.prob(s[8 * g + e], m_use);
        ls += pr;
        pe[e] = pr * scale_of(((vs[2 * g + (e >> 2)] >> (8 * (e & 3))) & 0xffu) + 7);
        // (a key that is not seen weighs nothing, whatever stands in the scale's place)
        if (MASK) pe[e] = pr > 0.f ? pe[e] : 0.f;
      }
      const bf16x8 pv = __builtin_convertvector(pe, bf16x8);
#pragma unroll
      for (int db = 0; db < Rows::kDBlocks; ++db) {
        const uint2 lo = dequantise4(raw[g][db][0], 0x1p-7f), hi = dequantise4(raw[g][db][1], 0x1p-7f);
        const bf16x8 v = __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
        rb.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pv, rb.o[db], 0, 0, 0);
      }
    }
    rb.add_to_sum(ls);
  }
};

// ---------------------------------------------------------------- the kernel

// 4 elements of a result, `i` counted in elements.
__device__ __forceinline__ void store_out(void* to, int64_t i, const f32x4& v, bool as_bf16) {
  if (as_bf16)
    store4(static_cast<__bf16*>(to) + i, v);
  else
    store4(static_cast<float*>(to) + i, v);
}

// The pages of a wavefront's blocks, 32 blocks at a time: one vector load, two lanes a block.  (Read
// block by block, each pair of ids is a trip to memory that the block's own loads wait for.)
struct BlockPages {
  int ids;
  // blocks b, b + kWaves, ... of the walk
  __device__ __forceinline__ void load(const int32_t* table, const KeyWalk& w, int b, int lane) {
    const int at = min(b + (lane >> 1) * kWaves, w.n - 1);
    ids = table[KeyRange(w, w.first_tokens(at)).page_index(w.tile(at) * 32 + (lane & 1) * kPageSize)];
  }
  __device__ __forceinline__ void get(int i, int (&page)[2]) const {
    page[0] = __builtin_amdgcn_readlane(ids, 2 * i);
    page[1] = __builtin_amdgcn_readlane(ids, 2 * i + 1);
  }
};

// A workgroup owns the 32 rows or fewer (token, head in group) of one KV head and a range of their
// walk, in blocks of 32 keys.  Its 4 wavefronts take the range's blocks in turn, each with a softmax
// of its own over a ring of its own, so that no barrier holds the stream up; their four states are
// joined through LDS, those of ranges by split_merge_kernel.
// Bound by memory: 64 decodes of 4K median at 32/8 heads, d 128, over the 8-bit cache stream 655 MB in
// 109 us, behind a window of 4096 over the bf16 cache 956 MB in 162 us (6.0 and 5.9 TB/s; a large copy
// reaches 5.1 on the same card).  The matrix pipes are busy 17 % and 9 % of the time.
//
// STAGES blocks of every wavefront are in flight while it waits for the first of them.  The loads are
// non-temporal (see async_stream16), also where sequences share their keys: looking that up in the page
// table, and a second copy of the walk for it, take 64 decodes that share 8192 keys over the 8-bit cache
// from 114 to 115 us and behind a window of 4096 from 82 to 74, and 64 that share none from 182 to 184.
// (Behind a window sequences share what they read only until they are a window past their common prefix:
// of a server's decodes the few.)
// (launched with 256 threads; the bound: see decode_kernel)
template <int D, class Block, int STAGES>
__global__ void __launch_bounds__(2 * kThreads) key_walk_kernel(const WalkArgs args) {
  constexpr int kWaveBytes = STAGES * Block::kBytes;
  constexpr int kCombineBytes = kWaves * 32 * (D + 2) * 4;
  __shared__ __attribute__((aligned(1024))) char
      lds[kWaves * kWaveBytes > kCombineBytes ? kWaves * kWaveBytes : kCombineBytes];
  using Rows = typename Block::Rows;

  const SeqDesc* descs = args.inline_descs;
  const int lane = threadIdx.x & 63;
  const int seq = find_seq_slot(descs, args.n_seq, blockIdx.x);
  const SeqDesc sd = uniform(descs[seq]);
  const KeySplitItem it = key_split_item(sd, blockIdx.x - sd.work_start, args.h_kv);
  const int split = it.split, kv_head = it.kv_head;

  const int gqa = args.h_q / args.h_kv;
  const int n_rows = sd.chunk_len * gqa;  // <= 32
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;

  const KeyWalk walk = make_walk(sd.prefix_len, sd.prefix_len + sd.chunk_len - 1, args.window, 32);
  const int b_first = split * sd.tiles_per_split * kWaves + wave;
  const int b_end = min(walk.n, (split + 1) * sd.tiles_per_split * kWaves);
  const int n_blocks = b_end > b_first ? (b_end - b_first + kWaves - 1) / kWaves : 0;
  const int n_full = min(n_blocks, max(0, walk.n_full - b_first + kWaves - 1) / kWaves);
  BlockPages pages;
  pages.load(args.page_table + sd.pt_off, walk, b_first, lane);

  Rows rb;
  rb.init(fabsf(args.scale_log2), lane);
  const bool valid = col < n_rows;
  const int rr = valid ? col : n_rows - 1;
  const int tok = rr / gqa;
  const int hq = kv_head * gqa + rr % gqa;
  rb.mask.position = sd.prefix_len + tok;
  rb.mask.window = args.window;
  Block::load_q(rb, args, args.q + ((int64_t)(sd.q_row + tok) * args.h_q + hq) * D, valid, half);
  Block block;
  block.init(lane);

  char* ring = lds + wave * kWaveBytes;
  const uint32_t ring_lds = lds_address(lds) + wave * kWaveBytes;
  // block i of the wavefront
  auto issue = [&](int i, int st) {
    if (i > 0 && i % 32 == 0)
      pages.load(args.page_table + sd.pt_off, walk, b_first + i * kWaves, lane);
    int page[2];
    pages.get(i & 31, page);
    const int b = b_first + i * kWaves, key0 = walk.tile(b) * 32;
    const KeyRange range(walk, walk.first_tokens(b));
    const uint32_t to = ring_lds + st * Block::kBytes;
    if (i < n_full)
      block.template issue<true, true>(args, page, range, key0, kv_head, to);
    else
      block.template issue<false, true>(args, page, range, key0, kv_head, to);
  };
  int st_issue = 0, st = 0;
  auto next = [](int x) { return x + 1 == STAGES ? 0 : x + 1; };
  for (int i = 0; i < STAGES - 1 && i < n_blocks; ++i) {
    issue(i, st_issue);
    st_issue = next(st_issue);
  }
  int i = 0;
  // (a loop each: with both forms of the step in one, 12 registers of the two-stage bf16 form spill, and
  // the wait for a reload is one for all loads in flight: 16 decodes of 354 at 32/8 heads 16.6 us, 26.9 so)
  auto blocks_to = [&](int end, auto mask_tag) {
    constexpr bool MASK = decltype(mask_tag)::value;
    for (; i < end; ++i) {
      if (i + STAGES - 1 < n_blocks) {
        issue(i + STAGES - 1, st_issue);
        st_issue = next(st_issue);
        wait_vmcnt<(STAGES - 1) * Block::kLoads>();  // the younger blocks may still fly
      } else {
        wait_vmcnt<0>();
      }
      const int b = b_first + i * kWaves, key0 = walk.tile(b) * 32;
      if (MASK) rb.mask.visit(walk.first_tokens(b), key0, half);
      block.template step<MASK>(rb, ring + st * Block::kBytes, key0);
      st = next(st);
      // every LDS read of the stage has returned before a load refills it
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  };
  blocks_to(n_full, std::false_type{});
  blocks_to(n_blocks, std::true_type{});

  // Combine the 4 wavefronts' (m, l, O) over their disjoint keys through LDS.
  const bool direct = sd.n_split == 1;
  void* o_base = direct ? args.out : args.part_o;
  float* l_base = direct ? args.lse : args.part_lse;
  const bool as_bf16 = direct && args.out_bf16;
  const int64_t row_base =
      direct ? (int64_t)sd.out_row : (int64_t)sd.part_row + (int64_t)split * sd.chunk_len;
  __syncthreads();  // all rings are drained and read
  float* sm_o = reinterpret_cast<float*>(lds);  // [wave][32][D]
  float* sm_ml = sm_o + kWaves * 32 * D;        // [wave][32][2]
  const float lt = rb.row_sum();
  if (valid) {
    float* op = sm_o + (wave * 32 + col) * D + 4 * half;
#pragma unroll
    for (int db = 0; db < Rows::kDBlocks; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = rb.o[db][4 * i + j];
        *reinterpret_cast<f32x4*>(op + db * 32 + 8 * i) = v;
      }
    if (half == 0) {
      sm_ml[(wave * 32 + col) * 2 + 0] = rb.m;
      sm_ml[(wave * 32 + col) * 2 + 1] = lt;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n_rows * (D / 4); e += kThreads) {
    const int rl = e / (D / 4), d4 = e % (D / 4);
    float mw[kWaves], lw[kWaves], mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      mw[w] = sm_ml[(w * 32 + rl) * 2 + 0];
      lw[w] = sm_ml[(w * 32 + rl) * 2 + 1];
      mm = fmaxf(mm, mw[w]);
    }
    // (a wavefront without a key has the sum 0; a NaN among a row's keys reaches its result)
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float lt_all = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (lw[w] == 0.f) continue;
      const float a = fast_exp2(mw[w] - mm);
      lt_all += a * lw[w];
      acc += *reinterpret_cast<const f32x4*>(sm_o + (w * 32 + rl) * D + d4 * 4) * a;
    }
    const float inv = lt_all != 0.f ? 1.f / lt_all : 0.f;
    const int64_t orow = (row_base + rl / gqa) * args.h_q + kv_head * gqa + rl % gqa;
    store_out(o_base, orow * D + d4 * 4, acc * inv, as_bf16);
    if (d4 == 0) l_base[orow] = lt_all != 0.f ? (mm + fast_log2(lt_all)) * kLn2 : -INFINITY;
  }
}

// ---------------------------------------------------------------- row-split

// The 64-key visits of a walk, for run_tiles(): a tile's number, or its complement where it is visited
// for first tokens.
struct WalkKeys {
  static constexpr bool kKept = true;  // a tile found when its page is looked up is kept for its loads
  KeyWalk w;
  WholeTiles whole_tiles;
  __device__ __forceinline__ explicit WalkKeys(const KeyWalk& walk) : w(walk), whole_tiles(walk) {}
  __device__ __forceinline__ int tile(int i) const {
    const int t = w.tile(i);
    return w.first_tokens(i) ? ~t : t;
  }
  __device__ __forceinline__ int key0(int v) const { return (v < 0 ? ~v : v) * 64; }
  __device__ __forceinline__ bool whole(int v) const { return whole_tiles.holds(v); }
  __device__ __forceinline__ int page_index(int v, int row) const {
    return KeyRange(w, v < 0).page_index(key0(v) + (row & ~(kPageSize - 1)));
  }
  __device__ __forceinline__ int slot(int v, int row) const {
    return KeyRange(w, v < 0).key(key0(v) + row) & (kPageSize - 1);
  }
  __device__ __forceinline__ void show(WindowMask& mask, int v, int half) const {
    mask.visit(v < 0, key0(v), half);
  }
};

// ---------------------------------------------------------------- row-split, 8-bit cache

// As ring_barrier(), and this wavefront's LDS writes are done.
template <int N>
__device__ __forceinline__ void ring_barrier_written() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The workgroup's LDS: stages of K and V tiles as they come, D bytes a row, of scale bytes, and two V
// tiles in bf16.  The long ring has 4 stages of each; the short one 3, and 2 for V, whose loads then
// stay a tile behind: at head dim 128 two workgroups of 4 wavefronts fit a compute unit.
template <int D, int NW, bool SHORT>
struct Fp8Ring {
  static constexpr int kStages = SHORT ? 3 : 4, kVStages = SHORT ? 2 : 4;
  static constexpr int kLag = SHORT ? 1 : 0, kRound = SHORT ? 6 : 4;
  static constexpr int kTile = 64 * D;  // K (or V) tile
  static constexpr int kScales = NW * 256;  // a wavefront's 64 lanes' worth
  static constexpr int kV = kStages * kTile, kS = kV + kVStages * kTile;
  static constexpr int kV16 = kS + kStages * kScales;
  static constexpr int kBytes = kV16 + 2 * (2 * kTile);
  static constexpr int kLdsBytes = kBytes > NW * 32 * D * 4 ? kBytes : NW * 32 * D * 4;  // (write_rows)
  // a tile's load instructions, 1 KiB each: every wavefront takes as many of K as of V, or, where
  // there are fewer of each than wavefronts, the first half of the wavefronts K and the others V
  static constexpr int kInstr = kTile / 1024, kRowsPerInstr = 1024 / D;
  static constexpr bool kBoth = kInstr >= NW;
  static constexpr int kPerWave = kBoth ? kInstr / NW : 1;
  static constexpr int kTileLoads = (kBoth ? 2 * kPerWave : 1) + 1;  // of K, V and scale bytes
  static_assert(kBoth || !SHORT, "V loads of their own");
  // loads of an iteration that its successor's barrier leaves in flight, and those of the prologue
  // behind the first tile's
  static constexpr int kYoungest = SHORT ? kPerWave + 1 : kTileLoads;
  static constexpr int kBehindFirst = kYoungest + kTileLoads;
  // the scale bytes of page p of a tile are where its first wavefront put them
  static constexpr int kScaleStride = kBoth ? NW / 4 * 256 : 256;
  // V rows a wavefront turns into bf16, and its lanes' bytes of them
  static constexpr int kRowsPerWave = 64 / NW, kLaneBytes = kRowsPerWave * D / 64;
};

// Rows of one wavefront of a chunk with what the tile walk needs of them.  A lane turns its pieces of a
// key into bf16, scale and all, as it reads them: exact, and the scores are sums in fp32.  (The matrix
// instructions that take 8 bits as they are keep some 13 bits below their largest product: with two
// channels whose products of 512 cancel, scores and LSE were off by 4e-3.  They save 64 conversions a
// tile: 2048 tokens at 32768, 32/8 heads, d 128, 948 us instead of 1000.)
template <int D, int NW, bool SHORT>
struct TileRows8 : RowBlock<D, WindowMask> {
  using Base = RowBlock<D, WindowMask>;
  using R = Fp8Ring<D, NW, SHORT>;
  static constexpr int kPieces = D / 32;
  int k8_off[kPieces];  // this lane's 16-byte pieces of key row `col`, within a K tile
  int ks_off;           // its scale byte within a stage's

  __device__ __forceinline__ void init(float scale, int ln) {
    Base::init(scale, ln, R::kV16);
    const int col = ln & 31, half = ln >> 5;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      k8_off[i] = col * D + swz8<D>(col, (i >> 1) * 4 + half * 2 + (i & 1)) * 16;
    ks_off = (col >> 4) * R::kScaleStride + (col & 15);
  }

  // Slot i: key block i & 1, slice i >> 1, of which two make a piece.
  struct KSide {
    const TileRows8& rb;
    const char* k_lds;
    const char* scales;
    float ks[2];
    uint4 raw[2][2];
    __device__ __forceinline__ KSide(const TileRows8& rows, const char* k, const char* s)
        : rb(rows), k_lds(k), scales(s) {}
    __device__ __forceinline__ void read(int i) {
      const int kb = i & 1, piece = i >> 2;
      if (i < 2) ks[kb] = scale_of((uint8_t)scales[rb.ks_off + kb * 2 * R::kScaleStride]);
      if (!(i & 2)) raw[kb][piece & 1] = *reinterpret_cast<const uint4*>(k_lds + kb * 32 * D + rb.k8_off[piece]);
    }
    __device__ __forceinline__ bf16x8 operand(int i) const {
      const uint4& x = raw[i & 1][(i >> 2) & 1];
      return __builtin_bit_cast(bf16x8, dequantise8(i & 2 ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y), ks[i & 1]));
    }
    template <int i>
    __device__ __forceinline__ void multiply(f32x16 (&s)[2]) {
      s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(i), rb.q[i >> 1], s[i & 1], 0, 0, 0);
    }
  };

  // The scores of a tile alone.
  __device__ __forceinline__ void qk(const char* k_lds, const char* scales, f32x16 (&s)[2]) const {
    KSide k(*this, k_lds, scales);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
    auto slot = [&](auto i) {
      k.read(decltype(i)::value);
      k.template multiply<decltype(i)::value>(s);
    };
    static_for<2 * Base::kSlices>(slot);
  }
};

// This wavefront's share of a tile's loads.
template <int D, int NW, bool SHORT>
struct Fp8Loader {
  using R = Fp8Ring<D, NW, SHORT>;
  uint32_t k_off[R::kPerWave], v_off[R::kPerWave];  // within the (page, KV head) block
  int row0, r_in, pos;
  bool values;  // !kBoth: this wavefront loads V

  __device__ __forceinline__ void init(int wave, int lane) {
    row0 = R::kBoth ? wave * R::kRowsPerWave : (wave & 3) * kPageSize;
    values = !R::kBoth && wave >= 4;
    r_in = lane / (D / 16);
    pos = lane % (D / 16);
#pragma unroll
    for (int j = 0; j < R::kPerWave; ++j) {
      const int row = row0 + j * R::kRowsPerInstr + r_in;
      k_off[j] = (row & 15) * D + swz8<D>(row, pos) * 16;
      v_off[j] = (row & 15) * D + pos * 16;
    }
  }
  // Loads K rows and scale bytes (K), V rows (V) of a tile into stages of the ring.
  template <bool K, bool V, class Keys>
  __device__ __forceinline__ void issue(const WalkArgs& args, int page, int tile, const Keys& keys,
                                        int kv_head, uint32_t ring, int k_stage, int v_stage, int wave,
                                        int lane) const {
    const int64_t block = (int64_t)page * args.h_kv + kv_head;
    const char* kp = args.k_pool + block * (kPageSize * D);
    const char* vp = args.v_pool + block * (kPageSize * D);
    const uint32_t k_to = ring + k_stage * R::kTile, v_to = ring + R::kV + v_stage * R::kTile;
    auto load = [&](uint32_t ko, uint32_t vo, int j) {
      const uint32_t at = (row0 + j * R::kRowsPerInstr) * D;
      if constexpr (R::kBoth) {
        if (K) async_load16<false>(kp, ko, k_to + at);
        if (V) async_load16<false>(vp, vo, v_to + at);
      } else {
        async_load16<false>(values ? vp : kp, values ? vo : ko, (values ? v_to : k_to) + at);
      }
    };
    if (keys.whole(tile)) {
#pragma unroll
      for (int j = 0; j < R::kPerWave; ++j) load(k_off[j], v_off[j], j);
    } else {
#pragma unroll
      for (int j = 0; j < R::kPerWave; ++j) {
        const int row = row0 + j * R::kRowsPerInstr + r_in;
        const int slot = keys.slot(tile, row);
        load(slot * D + swz8<D>(row, pos) * 16, slot * D + pos * 16, j);
      }
    }
    if (K)
      async_load4(args.scale + block * kScaleBytesPerPage, (lane & 7) * 4,
                  ring + R::kS + k_stage * R::kScales + wave * 256);
  }
};

// The wavefront's V rows of a tile, from 8 bits to bf16 where the transposing reads expect them.
template <int D, int NW, bool SHORT>
struct Fp8Convert {
  using R = Fp8Ring<D, NW, SHORT>;
  static constexpr int kWords = R::kLaneBytes / 4;
  static constexpr int kPieces = kWords > 4 ? kWords / 4 : 1;  // of 16 bytes (or one of 8)
  static constexpr int kPieceRows = kWords > 4 ? R::kRowsPerWave / kPieces : R::kRowsPerWave;
  static constexpr int kPieceWords = kWords / kPieces;
  int in_off, out_off, row;
  uint32_t raw[kWords];
  float scale[kPieces];
  uint2 half;

  __device__ __forceinline__ void init(int wave, int lane) {
    constexpr int kLanesPerRow = D / (4 * kPieceWords);
    row = wave * R::kRowsPerWave + lane / kLanesPerRow;
    const int at = lane % kLanesPerRow * kPieceWords;  // word of the row: 4 elements
    in_off = R::kV + row * D + at * 4;
    out_off = R::kV16 + row * (D * 2) + Swz<D>::v(row, at / 2) * 16;
  }
  // WHOLE: all keys of the tile are read.
  template <bool WHOLE, class Keys>
  __device__ __forceinline__ void read(const char* lds, int s_stage, int v_stage, int tile,
                                       const Keys& keys) {
    const char* in = lds + v_stage * R::kTile + in_off;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int r = row + p * kPieceRows;
      const char* s = lds + R::kS + s_stage * R::kScales + (r >> 4) * R::kScaleStride + kPageSize;
      scale[p] = scale_of((uint8_t)s[WHOLE ? r & 15 : keys.slot(tile, r)]);
      if constexpr (kPieceWords == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(in + p * kPieceRows * D);
        raw[4 * p] = x.x; raw[4 * p + 1] = x.y; raw[4 * p + 2] = x.z; raw[4 * p + 3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(in);
        raw[0] = x.x; raw[1] = x.y;
      }
    }
  }
  // word w of the lane's, written out behind every second one
  template <int w>
  __device__ __forceinline__ void convert(char* lds, int v16_stage) {
    const uint2 x = dequantise4(raw[w], scale[w / kPieceWords]);
    if constexpr (w % 2 == 0) {
      half = x;
    } else {
      constexpr int p = w / kPieceWords, c = w % kPieceWords / 2;
      *reinterpret_cast<uint4*>(lds + v16_stage * (2 * R::kTile) + out_off + p * kPieceRows * (D * 2) +
                                c * 16) = make_uint4(half.x, half.y, x.x, x.y);
    }
  }
};

// Walks tiles [kt_a, kt_b) of a walk, those below kt_mid without a mask: run_tiles() over the 8-bit
// cache.  At the barrier that opens iteration cur, K tile cur+1 and V tile cur+1 have landed as they
// are and V tile cur is there in bf16; in the iteration every wavefront turns its rows of V tile cur+1
// into bf16, beside the softmax of tile cur, and issues K tile cur+3 and V tile cur+3 (cur+2 with the
// short ring).
template <int D, int NW, bool SHORT, class Keys>
__device__ __forceinline__ void run_tiles8(TileRows8<D, NW, SHORT>& rb, const WalkArgs& args,
                                           ConstI32Ptr pt, int kt_a, int kt_mid, int kt_b,
                                           const Keys& keys, int kv_head, char* lds, int wave,
                                           int lane) {
  using R = Fp8Ring<D, NW, SHORT>;
  using Rows = TileRows8<D, NW, SHORT>;
  using Convert = Fp8Convert<D, NW, SHORT>;
  constexpr int kRound = R::kRound;
  static_assert(kWarmTiles % kRound == 0, "the walk's head is a whole number of ring rounds");
  if (kt_a >= kt_b) return;
  const int half = lane >> 5;
  const int last = kt_b - 1;
  const int kt_u = kt_mid >= kt_b ? kt_b : kt_a + (kt_mid - kt_a) / kRound * kRound;
  const uint32_t ring = lds_address(lds);
  Fp8Loader<D, NW, SHORT> ld;
  ld.init(wave, lane);
  Convert cv;
  cv.init(wave, lane);
  // the next tile and its page's id, and those before it
  int tile_next = 0, page_next = 0, tile_1 = 0, page_1 = 0;
  auto next_page = [&](int i) {
    if (SHORT) {
      page_1 = page_next;
      tile_1 = tile_next;
    }
    tile_next = keys.tile(min(i, last));
    page_next = pt[__builtin_amdgcn_readfirstlane(keys.page_index(tile_next, ld.row0))];
  };
  // the next K tile, and the V tile kLag before it if v_stage is one (with the short ring first: the
  // wait for it leaves K in flight)
  auto issue = [&](int k_stage, int v_stage) {
    if constexpr (SHORT) {
      if (v_stage >= 0)
        ld.template issue<false, true>(args, page_1, tile_1, keys, kv_head, ring, 0, v_stage, wave, lane);
      ld.template issue<true, false>(args, page_next, tile_next, keys, kv_head, ring, k_stage, 0, wave,
                                     lane);
    } else {
      ld.template issue<true, true>(args, page_next, tile_next, keys, kv_head, ring, k_stage, v_stage,
                                    wave, lane);
    }
  };
  auto k_stage = [&](int s) { return lds + s * R::kTile; };
  auto scales = [&](int s) { return lds + R::kS + s * R::kScales; };
  // prologue: K tiles kt_a .. kt_a+2 and V tiles up to kt_a+2-kLag
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    next_page(kt_a + i);
    issue(i, i - R::kLag);
  }
  next_page(kt_a + 3);
  f32x16 s0[2], s1[2];
  forget(s0);
  forget(s1);
  ring_barrier<R::kBehindFirst>();  // tile kt_a has landed, for everyone
  auto convert_all = [&](auto w) { cv.template convert<decltype(w)::value>(lds, 0); };
  cv.template read<false>(lds, 0, 0, keys.tile(kt_a), keys);
  static_for<Convert::kWords>(convert_all);
  rb.qk(k_stage(0), scales(0), s0);
  if (kt_u > kt_a) {
    float mx = -INFINITY;
#pragma unroll
    for (int f = 0; f < 32; ++f) mx = fmaxf(mx, s0[f >> 4][f & 15]);
    rb.template update_reference<false>(mx);
  }
  auto round = [&](int kt, auto mask, auto spec) {
    constexpr bool kMask = decltype(mask)::value, kSpeculate = decltype(spec)::value;
    auto iteration = [&](auto s_const) {
      constexpr int s = decltype(s_const)::value;
      constexpr int k_next = (s + 1) % R::kStages, v_next = (s + 1) % R::kVStages;
      const int cur = kt + s;
      if (cur < last) {
        ring_barrier_written<R::kYoungest>();
        auto at_slot = [&](auto slot) {
          constexpr int i = decltype(slot)::value;
          constexpr int kFirst = 6, kStep = D == 128 ? 2 : 1;
          // (up to a round's last iteration the next tile has the round's form)
          if constexpr (i == 1)
            cv.template read<!kMask && s + 1 < kRound>(lds, k_next, v_next, keys.tile(cur + 1), keys);
          if constexpr (i == Rows::kLoadSlot) {
            asm volatile("" : "+s"(page_next));  // the page id is first needed here, not before
            issue((s + 3) % R::kStages, (s + 3 - R::kLag) % R::kVStages);
          }
          if constexpr (i >= kFirst && (i - kFirst) % kStep == 0 &&
                        (i - kFirst) / kStep < Convert::kWords)
            cv.template convert<(i - kFirst) / kStep>(lds, (s + 1) & 1);
        };
        const typename Rows::KSide next(rb, k_stage(k_next), scales(k_next));
        const char* v_cur = lds + (s & 1) * (2 * R::kTile);  // + the bias in rb.v_off
        if constexpr (kMask) keys.show(rb.mask, keys.tile(cur), half);
        if constexpr (s & 1)
          rb.template fused<kMask, true, kSpeculate>(next, v_cur, s1, s0, keys.key0(keys.tile(cur)), half, at_slot);
        else
          rb.template fused<kMask, true, kSpeculate>(next, v_cur, s0, s1, keys.key0(keys.tile(cur)), half, at_slot);
        // (the scalar load goes here: see run_tiles)
        __builtin_amdgcn_sched_barrier(0);
        next_page(cur + 4);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    static_for<kRound>(iteration);
  };
  int kt = kt_a;
  const int end_u = min(kt_u, last);
  for (; kt < end_u && kt < kt_a + kWarmTiles; kt += kRound)
    round(kt, std::false_type{}, std::false_type{});
  for (; __builtin_expect_with_probability(kt < end_u, 1, 0.995); kt += kRound)
    round(kt, std::false_type{}, std::true_type{});
  for (; kt < last; kt += kRound) round(kt, std::true_type{}, std::false_type{});
  ring_barrier_written<R::kYoungest>();  // the last V tile is there in bf16, for everyone
  auto final_tile = [&](auto mask) {
    constexpr bool kMask = decltype(mask)::value;
    const typename Rows::KSide none(rb, nullptr, nullptr);
    const char* v_last = lds + ((last - kt_a) & 1) * (2 * R::kTile);
    if constexpr (kMask) keys.show(rb.mask, keys.tile(last), half);
    if ((last - kt_a) & 1)
      rb.template fused<kMask, false, false>(none, v_last, s1, s0, keys.key0(keys.tile(last)), half,
                                                   [](auto) {});
    else
      rb.template fused<kMask, false, false>(none, v_last, s0, s1, keys.key0(keys.tile(last)), half,
                                                   [](auto) {});
  };
  if (kt_u == kt_b)
    final_tile(std::false_type{});
  else
    final_tile(std::true_type{});
  ring_barrier<0>();
}

// Chunks: a workgroup of NW wavefronts owns NW * 32 query rows of one KV head and walks 64-key tiles,
// as prefill_kernel does, along the tiles of its rows' windows.
// SHORT: with the short ring, two workgroups to a compute unit.
// Bound by the matrix cores and the vector instructions of the softmax beside them: 2048 tokens at
// 32768 over the 8-bit cache (32/8 heads, d 128) take 1000 us, 1.13 PFLOP/s (counting 4 d a visible
// score; a large bf16 matrix product reaches 1.25), over the bf16 cache 951.  2048 tokens behind a window of 4096
// over the bf16 cache take 137 us, the matrix pipes and the vector units busy for 53 % of them each.
// Eight prompts of 1K median at d 64 behind a window of 1000 take 139 us, 29 % and 67 %: half the head
// dim leaves a score's softmax as it is, and walks of 18 tiles stay on run_tiles()'s exact route.
template <int D, int NW, bool kFp8, bool SHORT = false>
__global__ void __launch_bounds__(512) row_walk_kernel(const WalkArgs args) {
  constexpr int NV = SHORT ? 2 : 4;
  using Shape = PrefillShape<D, NW, NV>;
  using Rows = std::conditional_t<kFp8, TileRows8<D, NW, SHORT>, RowBlock<D, WindowMask>>;
  constexpr int kLdsBytes = kFp8 ? Fp8Ring<D, NW, SHORT>::kLdsBytes : Shape::kLdsBytes;
  __shared__ __attribute__((aligned(1024))) char lds[kLdsBytes];

  const SeqDesc* descs = args.inline_descs;
  const int seq = find_seq_slot(descs, args.n_seq, blockIdx.x);
  const SeqDesc sd = uniform(descs[seq]);
  const SlotItem it =
      row_split_item(sd, blockIdx.x - sd.work_start, args.h_kv, seq == args.n_seq - 1);
  if (!it.valid) return;
  const int kv_head = it.kv_head, split = it.split;

  const int gqa = args.h_q / args.h_kv;
  const int n_rows = sd.chunk_len * gqa;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int col = lane & 31, half = lane >> 5;

  Rows rb;
  if constexpr (kFp8)
    rb.init(fabsf(args.scale_log2), lane);
  else
    rb.init(fabsf(args.scale_log2), lane, Shape::kVBias);
  const int wg_row0 = it.row_tile * Shape::kRowsPerWg;
  const int r = wg_row0 + wave * 32 + col;
  const bool valid = r < n_rows;
  const int rr = valid ? r : (n_rows - 1);
  const int tok = rr / gqa;
  const int hq = kv_head * gqa + rr % gqa;
  rb.mask.position = sd.prefix_len + tok;
  rb.mask.window = args.window;
  const __bf16* qp = args.q + ((int64_t)(sd.q_row + tok) * args.h_q + hq) * D;
  std::conditional_t<kFp8, Fp8Block<D>, Bf16Block<D>>::load_q(rb, args, qp, valid, half);

  const int last_row = min(n_rows, wg_row0 + Shape::kRowsPerWg) - 1;
  const WalkKeys keys(make_walk(sd.prefix_len + wg_row0 / gqa, sd.prefix_len + last_row / gqa,
                                args.window, 64));
  const int kt_begin = split * sd.tiles_per_split;
  const int kt_end = min(keys.w.n, kt_begin + sd.tiles_per_split);
  const int kt_mid = max(kt_begin, min(kt_end, keys.w.n_full));
  ConstI32Ptr pt = (ConstI32Ptr)(args.page_table + sd.pt_off);
  if constexpr (kFp8) {
    run_tiles8<D, NW, SHORT>(rb, args, pt, kt_begin, kt_mid, kt_end, keys, kv_head, lds, wave, lane);
  } else {
    const Ring stages{lds, lds_address(lds)};
    TileLoader<D, NW> loader;
    loader.init(wave, lane);
    run_tiles<D, NW, NV, false>(rb, args, pt, kt_begin, kt_mid, kt_end, keys, kv_head, stages, loader,
                                wave, lane);
  }

  const bool direct = sd.n_split == 1;
  void* o_base = direct ? args.out : args.part_o;
  float* l_base = direct ? args.lse : args.part_lse;
  const int64_t row_base =
      direct ? (int64_t)sd.out_row : (int64_t)sd.part_row + (int64_t)split * sd.chunk_len;
  // (a range without a tile has the sum 0; a NaN among a row's keys reaches its result)
  const float lt = rb.row_sum();
  const float inv = lt != 0.f ? 1.f / lt : 0.f;
  const float lse = lt != 0.f ? (rb.m + fast_log2(lt)) * kLn2 : -INFINITY;
  if (valid && half == 0) l_base[(row_base + tok) * args.h_q + hq] = lse;
  if (direct && args.out_bf16)
    write_rows<D, NW, kLdsBytes>(rb, lds, inv, static_cast<__bf16*>(o_base), row_base, tok, hq,
                                        args.h_q, wg_row0, n_rows, wave, lane);
  else
    write_rows<D, NW, kLdsBytes>(rb, lds, inv, static_cast<float*>(o_base), row_base, tok, hq,
                                        args.h_q, wg_row0, n_rows, wave, lane);
}

}  // namespace medha
