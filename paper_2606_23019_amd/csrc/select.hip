// Choice of key blocks by a cheap score: means of blocks of tokens, and for every
// query block the topk key blocks whose mean key has the largest product with its
// mean query, as a Compressed Row Mask (and as the lists the attention kernel walks).
//
//   m_u = (1 / size_u) sum of the block's rows,  score_uv = sum_c qm_uc km_vc,
//   row u: the topk candidates of largest score (ties: the lowest v), and keep.
//
// A choice is a comparison, so the sums are held in 64 bits: neither the order of the
// sums nor an fp32 rounding decides between two blocks.  A mean is the fp32 rounding
// of the 64-bit sum's quotient, a score the 64-bit sum of exact products.
//
// Measured, 40 heads x 75600 tokens (591 x 591 blocks of 128, d = 128): means 113-118 us a
// tensor, 6.6-6.9 TB/s (2 GiB past the caches are read at 7.1); selection of 59 with kept
// blocks 122 us, 121-125 with candidates that leave half of the tiles (their bits cost what
// the skipped tiles save; scored all the same they took 145-150).  The products' 3.6 Gflop
// would take 54 at the 67 TFLOP/s of a large 64-bit matrix product.

#include <type_traits>

#include "device_common.h"
#include "launch.h"
#include "topk_border.h"

namespace sa {

namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

// ---- means ----
// One block of tokens a workgroup, d / 8 lanes a row, each lane 8 columns in 64 bits.
// Bound by the HBM bytes of x; a block's 8 to 32 KB are requested in one go.
struct MeansSide {
  const void* x;
  int64_t sb, sh, sn;
  float* means;
  int n_blk;
  int64_t items;
  bool stream;  // more than the last cache holds (40 heads x 75600 tokens: 133 -> 122 us)
};

template <int D, int BLK>
__device__ __forceinline__ void block_mean(const MeansSide& o, int64_t item, int H, int N) {
  constexpr int C = D / 8, R = 256 / C;  // rows a pass
  __shared__ double sums[4][D];
  const int64_t bh = item / o.n_blk;
  const int blk = (int)(item - bh * o.n_blk);
  const int lane = threadIdx.x & 63;
  const int chunk = threadIdx.x % C;
  const int size = min(BLK, N - blk * BLK);
  const int64_t sn = o.sn;
  const __bf16* from =
      (const __bf16*)o.x + (bh / H) * o.sb + (bh % H) * o.sh + (int64_t)blk * BLK * sn + 8 * chunk;
  u32x4 v[BLK / R];
  const int row0 = threadIdx.x / C;
  if (o.stream) {
#pragma unroll
    for (int i = 0; i < BLK / R; ++i)
      v[i] = row0 + i * R < size ? load_stream(from + (row0 + i * R) * sn) : u32x4{};
  } else {
#pragma unroll
    for (int i = 0; i < BLK / R; ++i)
      v[i] = row0 + i * R < size ? *(const u32x4*)(from + (row0 + i * R) * sn) : u32x4{};
  }
  double t[8] = {};
#pragma unroll
  for (int i = 0; i < BLK / R; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      t[2 * e] += (double)__uint_as_float(v[i][e] << 16);
      t[2 * e + 1] += (double)__uint_as_float(v[i][e] & 0xffff0000u);
    }
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int s = C; s < 64; s *= 2) t[e] += __shfl_xor(t[e], s, 64);
  if (lane < C)
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[threadIdx.x / 64][8 * chunk + e] = t[e];
  __syncthreads();
  if (threadIdx.x < D) {
    const int c = threadIdx.x;
    o.means[item * D + c] = (float)((sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c]) / size);
  }
}

// The blocks of one tensor, or of two (queries and keys) one after the other.
template <int D, int BLK0, int BLK1>
__global__ __launch_bounds__(256) void block_means_kernel(MeansSide first, MeansSide second, int H,
                                                          int N) {
  const int64_t item = blockIdx.x;
  if (item < first.items)
    block_mean<D, BLK0>(first, item, H, N);
  else
    block_mean<D, BLK1>(second, item - first.items, H, N);
}

// ---- selection ----
constexpr int kSelectLds = 156 * 1024;
constexpr int kSelectRows = 16;  // rows of a workgroup: one side of an MFMA tile

// Scores of `rows` (up to 16) query blocks against all key blocks by
// v_mfma_f64_16x16x4, as ordered keys in LDS, then a wavefront a row picks.  Lane l
// supplies row (or key block) l % 16 and, in step 4 s + e, the column 16 s + 4 (l / 16)
// + e of both sides, so that its loads are 16 bytes; every key block's sum runs in the
// same order, so equal blocks score alike.  16 key blocks that are no row's candidates are
// not scored at all (720p with frames that see the past: 368 -> 339 us); the candidate
// words are requested a tile ahead.
template <int D, int THREADS, bool CANDIDATES>
__global__ __launch_bounds__(THREADS) void block_select_kernel(SelectArgs a, int rows, int groups) {
  extern __shared__ uint64_t keys_all[];  // [rows][n_pad]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int waves = THREADS / 64;
  const int n_pad = (a.n_kb + 15) / 16 * 16;
  const int bh = blockIdx.x / groups;
  const int u0 = (blockIdx.x - bh * groups) * rows;
  const int n_rows = min(rows, a.n_qb - u0);
  const int l16 = lane & 15, g = lane >> 4;
  // Rows of a selection are of nearly one length, so the attention takes them in the
  // XCD layout with the heads in index order, with nothing to sort: a share of the
  // places here instead of the schedule's two launches.
  if (a.order) {
    const int64_t items = (int64_t)a.B * a.H * a.n_qb;
    const int64_t step = (int64_t)gridDim.x * THREADS;
    for (int64_t p = (int64_t)blockIdx.x * THREADS + threadIdx.x; p < items; p += step) {
      int u;
      const int unit = xcd_slice(p, a.B * a.H, a.n_qb, &u);
      a.order[p] = unit * a.n_qb + u;
    }
  }

  const int h = bh % a.H;
  const int words = (a.n_kb + 63) / 64;
  // the candidate bits of rows 4 i + l / 16 from key block v0 on, whose words hold 16 more
  uint64_t may[4] = {};
  auto load_candidates = [&](int v0) {
    const uint64_t* from = a.candidates + ((int64_t)(a.cand_per_batch ? bh : h) * a.n_qb + u0) * words;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      may[i] = v0 < a.n_kb ? from[min(4 * i + g, n_rows - 1) * words + v0 / 64] >> (v0 & 63) : 0;
  };
  if (CANDIDATES) load_candidates(wave * 16);

  const float* qrow = a.qm + ((int64_t)bh * a.n_qb + u0 + min(l16, n_rows - 1)) * D + 4 * g;
  const float* kmat = a.km + (int64_t)bh * a.n_kb * D + 4 * g;
  double qa[D / 4];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const f32x4 v = *(const f32x4*)(qrow + 16 * s);
#pragma unroll
    for (int e = 0; e < 4; ++e) qa[4 * s + e] = v[e];
  }
  for (int v0 = wave * 16; v0 < a.n_kb; v0 += waves * 16) {
    const int v = v0 + l16;
    uint64_t now[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) now[i] = may[i];
    if constexpr (CANDIDATES) {
      load_candidates(v0 + waves * 16);
      if (!__any(((now[0] | now[1] | now[2] | now[3]) & 0xffff) != 0)) {
        for (int row = g; row < n_rows; row += 4) keys_all[row * n_pad + v] = 0;
        continue;
      }
    }
    const float* krow = kmat + (int64_t)min(v, a.n_kb - 1) * D;
    f32x4 kb[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) kb[s] = *(const f32x4*)(krow + 16 * s);
    f64x4 c = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f64_16x16x4f64(qa[4 * s + e], (double)kb[s][e], c, 0, 0, 0);
    // register i of lane l holds row 4 i + l / 16 (64-bit tiles interleave rows), key block v
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * i + g;
      if (row < n_rows)
        keys_all[row * n_pad + v] = !CANDIDATES || ((now[i] >> l16) & 1ull) ? order_key(c[i]) : 0;
    }
  }
  __syncthreads();
  for (int row = wave; row < n_rows; row += waves) {
    const int64_t at = ((int64_t)bh * a.n_qb + u0 + row);
    const int64_t shared = ((int64_t)h * a.n_qb + u0 + row);
    // mask words, 64 at a time: lane l loads word w0 + l, and all take word i from lane i
    const uint64_t* keep = a.keep ? a.keep + (a.keep_per_batch ? at : shared) * words : nullptr;
    auto words_from = [&](const uint64_t* p, int w0) { return p && w0 + lane < words ? p[w0 + lane] : 0; };
    auto word_of = [](uint64_t mine, int i) {
      return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, i) |
             (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), i) << 32;
    };
    uint64_t* keys = keys_all + row * n_pad;
    uint64_t kept = words_from(keep, 0);
    Border edge;
    if (words <= 4)
      edge = border_of<4>(keys, a.n_kb, a.topk, lane);
    else if (words <= 10)
      edge = border_of<10>(keys, a.n_kb, a.topk, lane);
    else if (words <= 20)
      edge = border_of<20>(keys, a.n_kb, a.topk, lane);
    else
      edge = border_of_long(keys, a.n_kb, a.topk, lane);
    const uint64_t below = (1ull << lane) - 1ull;
    int done = 0;
    for (int w = 0; w < words; ++w) {
      const uint64_t key = 64 * w + lane < a.n_kb ? keys[64 * w + lane] : 0;
      uint64_t word = __ballot(key >= edge.lo);
      if (edge.ties >= 0) {
        const uint64_t same = __ballot(key == edge.lo);
        const bool first = key == edge.lo && (int)__popcll(same & below) < edge.ties;
        word = __ballot(key > edge.lo || first);
        edge.ties = max(0, edge.ties - (int)__popcll(same));
      }
      if (keep) {
        if (w > 0 && w % 64 == 0) kept = words_from(keep, w);
        const int real = a.n_kb - 64 * w;
        word |= word_of(kept, w % 64) & (real < 64 ? (1ull << real) - 1ull : ~0ull);
      }
      if (lane == 0) a.bits[at * words + w] = word;
      if (a.counts && ((word >> lane) & 1ull))
        a.lists[at * a.n_kb + done + __popcll(word & below)] = 64 * w + lane;
      done += __popcll(word);
    }
    if (a.counts && lane == 0) a.counts[at] = done;
  }
}

// Rows of a workgroup whose keys LDS holds, 0 where it does not hold one.
int rows_together(int n_kb) {
  const int64_t rows = kSelectLds / (((int64_t)n_kb + 15) / 16 * 16 * 8);
  return (int)(rows < kSelectRows ? rows : kSelectRows);
}

}  // namespace

bool block_means_fits(int64_t blocks) { return launchable(blocks, 256); }

hipError_t launch_block_means(const MeansArgs& q, const MeansArgs& k, int B, int H, int N, int d,
                              hipStream_t stream) {
  auto side = [&](const MeansArgs& a) {
    const int n_blk = (N + a.blk - 1) / a.blk;
    return MeansSide{a.x, a.sb, a.sh, a.sn, a.means, n_blk, a.x ? (int64_t)B * H * n_blk : 0,
                     (int64_t)B * H * N * d * 2 > kLastLevelCache};
  };
  const MeansSide first = side(q), second = side(k);
  if (!block_means_fits(first.items + second.items)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(first.items + second.items));
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, first, second, H, N);
  };
  const bool q128 = q.blk == 128, k128 = k.blk == 128;
  if (d == 128)
    q128 ? (k128 ? run(block_means_kernel<128, 128, 128>) : run(block_means_kernel<128, 128, 64>))
         : (k128 ? run(block_means_kernel<128, 64, 128>) : run(block_means_kernel<128, 64, 64>));
  else
    q128 ? (k128 ? run(block_means_kernel<64, 128, 128>) : run(block_means_kernel<64, 128, 64>))
         : (k128 ? run(block_means_kernel<64, 64, 128>) : run(block_means_kernel<64, 64, 64>));
  return hipGetLastError();
}

bool block_select_fits(int64_t heads, int n_qb, int n_kb) {
  const int64_t rows = rows_together(n_kb);
  return rows > 0 && launchable(heads * ((n_qb + rows - 1) / rows), 512);
}

hipError_t launch_block_select(const SelectArgs& a, hipStream_t stream) {
  if (!block_select_fits((int64_t)a.B * a.H, a.n_qb, a.n_kb)) return hipErrorInvalidValue;
  const int rows = rows_together(a.n_kb);
  const int groups = (a.n_qb + rows - 1) / rows;
  const int64_t grid = (int64_t)a.B * a.H * groups;
  const int lds = rows * ((a.n_kb + 15) / 16 * 16) * 8;
  // up to a workgroup a compute unit, 16 wavefronts: a row each (24 heads x 63 x 63 blocks
  // 10.6 -> 9.2 us); more workgroups share the units.  Groups of four rows on
  // v_mfma_f64_4x4x4 spread a small problem further (one group 13.6 -> 9.5 us) but read
  // the key blocks four times as often (5 heads x 256 x 256 blocks: 15.0 -> 16.4 us).
  const bool few = grid <= 256;
  auto pick = [&](auto candidates) {
    constexpr bool C = decltype(candidates)::value;
    return a.d == 128 ? (few ? block_select_kernel<128, 1024, C> : block_select_kernel<128, 512, C>)
                      : (few ? block_select_kernel<64, 1024, C> : block_select_kernel<64, 512, C>);
  };
  auto kernel = a.candidates ? pick(std::true_type{}) : pick(std::false_type{});
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)kernel,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(few ? 1024 : 512), lds, stream, a, rows, groups);
  return hipGetLastError();
}

}  // namespace sa
