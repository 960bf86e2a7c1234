// The border between a row's topk largest scores and the rest, found by one wavefront.
#pragma once

#include "device_common.h"

namespace sa {

// A double's bits, ordered as unsigned numbers: 0 no candidate, 1 NaN, then -inf up.
__device__ __forceinline__ uint64_t order_key(double x) {
  if (x != x) return 1;
  x += 0.0;  // -0 equals 0
  const uint64_t b = (uint64_t)__double_as_longlong(x);
  return (b >> 63) ? ~b : b | (1ull << 63);
}

// The border of a row: its keys of `lo` and above are the chosen ones, of those equal
// to `lo` the first `ties` only (negative: all of them).
struct Border {
  uint64_t lo;
  int ties;
};

// The wavefront bisects the key space for a border with exactly topk keys on it or
// above, one bit a step from the top; most rows have one as soon as the border's
// neighbours differ.  count(t) is the number of keys that are at least t.
template <typename Count>
__device__ __forceinline__ Border find_border(int topk, Count count) {
  if (count(1) <= topk) return {1, -1};  // every candidate
  uint64_t lo = 0;                       // count(lo) > topk
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t t = lo | (1ull << bit);
    const int n = count(t);
    if (n == topk) return {t, -1};
    if (n > topk) lo = t;
  }
  return {lo, topk - count(lo + 1)};  // no key is ~0
}

// With the keys, 64 a word, in registers: rows of up to 64 W.
template <int W>
__device__ __forceinline__ Border border_of(const uint64_t* keys, int n_kb, int topk, int lane) {
  uint64_t key[W];
#pragma unroll
  for (int w = 0; w < W; ++w) key[w] = 64 * w + lane < n_kb ? keys[64 * w + lane] : 0;
  return find_border(topk, [&](uint64_t t) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) n += __popcll(__ballot(key[w] >= t));
    return n;
  });
}

// Longer rows read them from LDS in every step.
__device__ __forceinline__ Border border_of_long(const uint64_t* keys, int n_kb, int topk, int lane) {
  return find_border(topk, [&](uint64_t t) {
    int n = 0;
    for (int v = lane; v < n_kb + lane; v += 64) n += __popcll(__ballot(v < n_kb && keys[v] >= t));
    return n;
  });
}

}  // namespace sa
