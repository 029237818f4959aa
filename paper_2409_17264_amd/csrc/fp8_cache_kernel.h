// The 8-bit KV cache for gfx950: a chunk's keys and values quantised as they are written into the
// paged pools, and read back.
//
// A row is one token's head_dim elements of one KV head.  It is held as e4m3 values and one scale
// 2^(byte - 127) for the row: with E the exponent field of the row's largest finite magnitude,
//     byte = max(E - 7, 10),   value = round to nearest even of x * 2^(127 - byte).
// The largest value then lies in [128, 256], so nothing saturates (e4m3 ends at 448); an element
// keeps its 4 significant bits down to 2^-13 of the largest, since e4m3 is itself a floating format,
// which is why a power of two costs no accuracy and a finer scale than one a row brings none.  With
// byte >= 10 every value times its scale is zero or a normal bf16 number: reading back is exact.
//
// Both kernels move bytes only and are bound by memory: 3 d + 1 bytes a row each for K and for V.
#pragma once

#include "common.h"

namespace medha {

constexpr int kScaleBytesPerPage = 2 * kPageSize;  // per KV head: the keys' 16 bytes, then the values'
constexpr int kLeastScaleByte = 10;

struct Fp8CacheArgs {
  uint4* k_rows;  // bf16 [rows][h_kv][d]: read by the append, written by the read
  uint4* v_rows;
  void* k_pool;
  void* v_pool;
  uint8_t* scale;
  const int32_t* page_table;
  int32_t n_seq;
  int32_t h_kv;
  int32_t words_per_row;  // of 16 elements (the append) or of 8 (the read), a lane's share
  int32_t num_pages;
  int32_t total_rows;
  int32_t reserved;
  AppendDesc descs[kMaxInlineSeq];
};
static_assert(sizeof(Fp8CacheArgs) <= 4096, "kernel argument block too large");

// Where word `idx` of a launch lives, counted in words: in the dense rows, in the pool, and its row's
// scale bytes.
struct Fp8Place {
  int64_t row_word, pool_word, scale_byte;
  int word;
  bool valid;
};

// All 64 lanes have to be active; those past the launch's end stand for its last word.
__device__ __forceinline__ Fp8Place fp8_place(const Fp8CacheArgs& args, int64_t idx, int64_t total) {
  const int per_token = args.h_kv * args.words_per_row;
  const int64_t at = min(idx, total - 1);
  const int row = (int)(at / per_token);
  const int rem = (int)(at % per_token);
  const int head = rem / args.words_per_row;
  Fp8Place p;
  p.word = rem % args.words_per_row;
  const int seq = find_last(args.n_seq, row, [&](int i) { return args.descs[i].row_rank; });
  const AppendDesc sd = args.descs[seq];
  const int j = row - sd.row_rank;
  const int t = sd.prefix_len + j;
  const int page = args.page_table[sd.pt_off + (t >> 4)];
  p.valid = (unsigned)page < (unsigned)args.num_pages;
  const int64_t page_head = (int64_t)page * args.h_kv + head;
  p.row_word = ((int64_t)(sd.src_row + j) * args.h_kv + head) * args.words_per_row + p.word;
  p.pool_word = (page_head * kPageSize + (t & 15)) * args.words_per_row + p.word;
  p.scale_byte = page_head * kScaleBytesPerPage + (t & 15);
  return p;
}

// The scale that a byte stands for.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Exponent byte of a row from one lane's 16 elements; the row's lanes (4 or 8 neighbours) agree.
// Infinities and NaN do not count: they become NaN, and the row's other elements keep their values.
__device__ __forceinline__ uint32_t row_scale_byte(uint4 x, uint4 y, int lanes) {
  uint32_t top = 0;
  for (uint32_t w : {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w})
    for (uint32_t h : {w & 0x7fffu, (w >> 16) & 0x7fffu}) top = max(top, h < 0x7f80u ? h : 0u);
  for (int m = 1; m < lanes; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  return max((int)(top >> 7) - 7, kLeastScaleByte);
}

// Two bf16 elements to e4m3 in the low or high half of `into`.  Finite magnitudes are held below
// 1.875 * 2^127, the largest that does not round up to 2^128, which bf16 could not read back.
template <bool HIGH>
__device__ __forceinline__ s16x2 quantise_pair(s16x2 into, uint32_t w, float scale) {
  uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
  lo = lo < 0x7f80u ? min(lo, 0x7f70u) : lo;
  hi = hi < 0x7f80u ? min(hi, 0x7f70u) : hi;
  w = (w & 0x80008000u) | lo | (hi << 16);
  return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(into, __builtin_bit_cast(bf16x2, w), scale, HIGH);
}

__device__ __forceinline__ uint2 quantise8(uint4 x, uint32_t byte) {
  const float scale = scale_of(byte);
  s16x2 lo = {0, 0}, hi = {0, 0};
  lo = quantise_pair<false>(lo, x.x, scale);
  lo = quantise_pair<true>(lo, x.y, scale);
  hi = quantise_pair<false>(hi, x.z, scale);
  hi = quantise_pair<true>(hi, x.w, scale);
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

__device__ __forceinline__ uint4 quantise16(uint4 x, uint4 y, uint32_t byte) {
  const uint2 a = quantise8(x, byte), b = quantise8(y, byte);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// 4 e4m3 values times their scale, as bf16.
__device__ __forceinline__ uint2 dequantise4(uint32_t x, float scale) {
  return make_uint2(
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true)));
}
__device__ __forceinline__ uint4 dequantise8(uint2 x, float scale) {
  const uint2 a = dequantise4(x.x, scale), b = dequantise4(x.y, scale);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// One lane per 16 elements of one (token, KV head), for K and for V, so that what it writes to the pools
// is 16 bytes (13291 tokens at 8 heads, d 128: 18.7 us with 8 elements a lane, 16.4 with 16: 5.0 TB/s).
// A page id outside [0, num_pages) is skipped: nothing outside the pools is ever written.
static __global__ void __launch_bounds__(kThreads) kv_append_fp8_kernel(const Fp8CacheArgs args) {
  const int64_t total = (int64_t)args.total_rows * args.h_kv * args.words_per_row;
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < total; first += step) {
    const int64_t idx = first + threadIdx.x;
    const Fp8Place p = fp8_place(args, idx, total);
    const uint4 k0 = args.k_rows[2 * p.row_word], k1 = args.k_rows[2 * p.row_word + 1];
    const uint4 v0 = args.v_rows[2 * p.row_word], v1 = args.v_rows[2 * p.row_word + 1];
    const uint32_t kb = row_scale_byte(k0, k1, args.words_per_row);
    const uint32_t vb = row_scale_byte(v0, v1, args.words_per_row);
    if (idx >= total || !p.valid) continue;
    static_cast<uint4*>(args.k_pool)[p.pool_word] = quantise16(k0, k1, kb);
    static_cast<uint4*>(args.v_pool)[p.pool_word] = quantise16(v0, v1, vb);
    if (p.word == 0) {
      args.scale[p.scale_byte] = (uint8_t)kb;
      args.scale[p.scale_byte + kPageSize] = (uint8_t)vb;
    }
  }
}

// The way back, one lane per 8 elements: 16 bytes written (32768 tokens at 8 heads, d 128: 42.2 us; with
// 16 elements a lane, whose stores leave half of every line to another instruction, 46.6).  Tokens of a
// page id outside [0, num_pages) read as zero.
// kOnce: rows that the last-level cache cannot hold until somebody reads them are stored
// non-temporally (65536 tokens 81.0 -> 73.7 us, with an append that reads them behind it 181 -> 173;
// 16384 tokens and their append 38.1 -> 41.7, 32768 81.2 -> 85.4: those are still in the cache).
template <bool kOnce>
__global__ void __launch_bounds__(kThreads) kv_read_fp8_kernel(const Fp8CacheArgs args) {
  const int64_t total = (int64_t)args.total_rows * args.h_kv * args.words_per_row;
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < total; first += step) {
    const int64_t idx = first + threadIdx.x;
    const Fp8Place p = fp8_place(args, idx, total);
    if (idx >= total) continue;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (p.valid) {
      k = dequantise8(static_cast<const uint2*>(args.k_pool)[p.pool_word],
                      scale_of(args.scale[p.scale_byte]));
      v = dequantise8(static_cast<const uint2*>(args.v_pool)[p.pool_word],
                      scale_of(args.scale[p.scale_byte + kPageSize]));
    }
    if (kOnce) {
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, k),
                                  reinterpret_cast<u32x4*>(args.k_rows + p.row_word));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v),
                                  reinterpret_cast<u32x4*>(args.v_rows + p.row_word));
    } else {
      args.k_rows[p.row_word] = k;
      args.v_rows[p.row_word] = v;
    }
  }
}

}  // namespace medha
