// The border between a row's topk largest scores and the rest, found by one wavefront.
#pragma once

#include <type_traits>

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

// Sum over the wavefront of a small number from each lane, in every lane.
__device__ __forceinline__ int wave_sum(int x) {
  auto dpp = [](int v, auto ctrl) {
    return v + __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, 0xF, 0xF, false);
  };
  x = dpp(x, std::integral_constant<int, 0xB1>{});   // lane ^ 1
  x = dpp(x, std::integral_constant<int, 0x4E>{});   // lane ^ 2
  x = dpp(x, std::integral_constant<int, 0x141>{});  // mirrored inside 8
  x = dpp(x, std::integral_constant<int, 0x140>{});  // mirrored inside 16
  auto r = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  x = (int)(r[0] + r[1]);
  r = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  return __builtin_amdgcn_readfirstlane((int)(r[0] + r[1]));
}

// Greatest of a word over the wavefront.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto dpp = [](uint32_t v, auto ctrl) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  x = dpp(x, std::integral_constant<int, 0xB1>{});
  x = dpp(x, std::integral_constant<int, 0x4E>{});
  x = dpp(x, std::integral_constant<int, 0x141>{});
  x = dpp(x, std::integral_constant<int, 0x140>{});
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(max(r[0], r[1]));
}

// The wavefront looks for a border with exactly topk keys on it or above, between one
// with more and one with fewer.  The upper words of the keys settle nearly all rows (20
// bits of the score's mantissa), in compares of half the width; the lower ones are
// looked at only where keys agree in the upper ones.  The largest scores lie within a
// few binades of the greatest, 2^20 words each, so with SEARCH the steps first go down
// from there by doubling distances and then halve the interval: some 12 steps for a row
// of 591, where bit by bit it takes 24 (selection at 720p, 40 heads x 591 x 591: 169 ->
// 152 us).  Rows of a few words go bit by bit: their steps cost less than the longer
// code (decode, 64 blocks: 5.6 us, 8.6 with SEARCH).  high(t) counts the keys whose upper
// word is at least t, low(h, t) those of upper word h whose lower word is at least t.
template <bool SEARCH, typename High, typename Low>
__device__ __forceinline__ Border find_border(int n_keys, int topk, uint32_t highest, High high,
                                              Low low) {
  if (n_keys <= topk) return {1, -1};  // every candidate
  // more than topk keys at h and above (all of them), fewer at `top` and above
  uint32_t h = 0, top = SEARCH ? highest + 1 : 0, gap = 1u << 20;
  if constexpr (!SEARCH) {
    for (uint32_t bit = 1u << 31; bit != 0; bit >>= 1) {
      const int n = high(h | bit);
      if (n == topk) return {(uint64_t)(h | bit) << 32, -1};
      if (n > topk) h |= bit;
    }
  }
  while (SEARCH && top - h > 1) {  // 12 steps down at most, every other one halves the interval
    uint32_t t = h + (top - h) / 2;
    if (h == 0 && gap != 0) {
      if (highest > gap && highest - gap > t && highest - gap < top) t = highest - gap;
      gap <<= 1;
    }
    const int n = high(t);
    if (n == topk) return {(uint64_t)t << 32, -1};
    if (n > topk)
      h = t;
    else
      top = t;
  }
  const int above = high(h + 1);
  uint32_t lo = 0;  // more than topk keys at (h, lo) and above
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t t = lo | (1u << bit);
    const int n = above + low(h, t);
    if (n == topk) return {(uint64_t)h << 32 | t, -1};
    if (n > topk) lo = t;
  }
  const int more = lo == ~0u ? 0 : low(h, lo + 1);
  return {(uint64_t)h << 32 | lo, topk - above - more};
}

// With the keys, 64 a word, in registers: rows of up to 64 W.
template <int W>
__device__ __forceinline__ Border border_of(const uint64_t* keys, int n_kb, int topk, int lane) {
  constexpr bool kFew = W <= 4;
  uint32_t hi[W], lo[W];
  int n = 0;
  uint32_t most = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const uint64_t key = 64 * w + lane < n_kb ? keys[64 * w + lane] : 0;
    hi[w] = (uint32_t)(key >> 32);
    lo[w] = (uint32_t)key;
    if (kFew) {
      n += __popcll(__ballot(key != 0));
    } else {
      n += key != 0;
      most = max(most, hi[w]);
    }
  }
  if (!kFew) {
    n = wave_sum(n);
    most = wave_max(most);
  }
  return find_border<!kFew>(
      n, topk, most,
      [&](uint32_t t) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += kFew ? (int)__popcll(__ballot(hi[w] >= t)) : hi[w] >= t;
        return kFew ? c : wave_sum(c);
      },
      [&](uint32_t h, uint32_t t) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += __popcll(__ballot(hi[w] == h && lo[w] >= t));
        return c;
      });
}

// Longer rows read them from LDS in every step.
__device__ __forceinline__ Border border_of_long(const uint64_t* keys, int n_kb, int topk, int lane) {
  auto count = [&](auto is) {
    int c = 0;
    for (int v = lane; v < n_kb; v += 64) c += is((uint32_t)(keys[v] >> 32), (uint32_t)keys[v]);
    return wave_sum(c);
  };
  uint32_t most = 0;
  for (int v = lane; v < n_kb; v += 64) most = max(most, (uint32_t)(keys[v] >> 32));
  return find_border<true>(
      count([](uint32_t h, uint32_t l) { return (h | l) != 0; }), topk, wave_max(most),
      [&](uint32_t t) { return count([=](uint32_t h, uint32_t) { return h >= t; }); },
      [&](uint32_t u, uint32_t t) { return count([=](uint32_t h, uint32_t l) { return h == u && l >= t; }); });
}

// The border of one row found by all WAVES wavefronts of a workgroup together, each with
// the keys of W words in registers: rows of up to 64 W WAVES.  `counts` is LDS of 2 x
// WAVES numbers; every thread calls this, and all get the border.
template <int W, int WAVES>
__device__ __forceinline__ Border group_border(const uint64_t* keys, int n_kb, int topk, int wave,
                                               int lane, int (*counts)[WAVES]) {
  uint32_t hi[W], lo[W];
  int n = 0;
  uint32_t most = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int v = 64 * (w * WAVES + wave) + lane;
    const uint64_t key = v < n_kb ? keys[v] : 0;
    hi[w] = (uint32_t)(key >> 32);
    lo[w] = (uint32_t)key;
    n += key != 0;
    most = max(most, hi[w]);
  }
  int turn = 0;  // the numbers of one call are read while those of the next are written
  auto gather = [&](int mine) {
    if (lane == 0) counts[turn][wave] = mine;
    __syncthreads();
    const int other = lane < WAVES ? counts[turn][lane] : 0;
    turn ^= 1;
    return other;
  };
  n = wave_sum(gather(wave_sum(n)));
  most = wave_max((uint32_t)gather((int)wave_max(most)));
  return find_border<true>(
      n, topk, most,
      [&](uint32_t t) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += hi[w] >= t;
        return wave_sum(gather(wave_sum(c)));
      },
      [&](uint32_t h, uint32_t t) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) c += hi[w] == h && lo[w] >= t;
        return wave_sum(gather(wave_sum(c)));
      });
}

}  // namespace sa
