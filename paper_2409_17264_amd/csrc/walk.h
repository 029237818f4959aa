// Which keys the rows of a workgroup see under a sliding window with first tokens that stay
// visible, and the order in which their tiles are walked.  Host and device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace medha {

// The row at position p sees key t if t <= p and (t > p - keys or t < sinks).
struct Window {
  int32_t keys = INT32_MAX;  // INT32_MAX: no window
  int32_t sinks = 0;
};

// The tiles of `tile_keys` keys that rows at positions [p_a, p_b] see, as one row of n visits.  A
// visit shows a row either the window's keys of its tile, or its first tokens that no window of the
// row reaches: every visit's keys are one interval for each row, and no key is shown twice.  (A tile
// that holds keys of both kinds is visited twice.)  The windows reach keys [lo, end), the visits for
// first tokens show keys [0, first).  Softmax attention does not care for the order of its keys, so
// the tiles that every row's window covers come first (n_full of them, which need no mask), behind
// them the other tiles up to the rows' own, the first tokens' and the left edge of the windows:
//     [u0, w1)  [0, s1)  [w0, u0)
struct KeyWalk {
  int32_t lo, end, first;
  int32_t w0, w1, u0, s1;
  int32_t n, n_full;

  __host__ __device__ __forceinline__ bool first_tokens(int i) const {
    return (uint32_t)(i - (w1 - u0)) < (uint32_t)s1;
  }
  __host__ __device__ __forceinline__ int tile(int i) const {
    const int rest = i - (w1 - u0);
    return rest < 0 ? u0 + i : rest < s1 ? rest : w0 + rest - s1;
  }
};

// 0 <= p_a <= p_b < 2^31 - 1.
__host__ __device__ inline KeyWalk make_walk(int32_t p_a, int32_t p_b, const Window& win,
                                             int32_t tile_keys) {
  const auto at_least_0 = [](int32_t x) { return x > 0 ? x : 0; };
  KeyWalk k;
  k.lo = at_least_0(p_a - win.keys + 1);
  k.end = p_b + 1;
  const int32_t all_see = at_least_0(p_b - win.keys + 1);  // from here on every row sees, up to p_a
  k.first = win.sinks < all_see ? win.sinks : all_see;
  k.w0 = k.lo / tile_keys;
  k.w1 = (k.end - 1) / tile_keys + 1;
  k.s1 = k.first > 0 ? (k.first - 1) / tile_keys + 1 : 0;
  const int32_t u0 = all_see > 0 ? (all_see - 1) / tile_keys + 1 : 0, u1 = (p_a + 1) / tile_keys;
  k.n_full = u1 > u0 ? u1 - u0 : 0;
  k.u0 = k.n_full > 0 ? u0 : k.w0;
  k.n = k.w1 - k.w0 + k.s1;
  return k;
}

// Whether every key of a visit's 64-key tile is read: `v` is a tile's number, or its complement where it
// is visited for first tokens.
struct WholeTiles {
  int32_t from;         // tiles whose every key the windows reach,
  uint32_t n, n_first;  // and of the first tokens'
  __host__ __device__ __forceinline__ explicit WholeTiles(const KeyWalk& w) {
    from = (int32_t)(((uint32_t)w.lo + 63) >> 6);  // (lo + 63 may pass 2^31 - 1)
    n = w.end >> 6 > from ? (w.end >> 6) - from : 0;
    n_first = w.first >> 6;
  }
  __host__ __device__ __forceinline__ bool holds(int32_t v) const {
    return (uint32_t)(v - from) < n || (uint32_t)v + n_first < n_first;
  }
};

}  // namespace medha
