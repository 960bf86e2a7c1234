// Attention of one query token a sequence over the blocks of its cache that a cheap
// score selects.
//
// For sequence b of length L (blocks 0 .. last, last = ceil(L / blk) - 1) and key head
// h, whose group holds G query heads:
//   score_v = <means_v, sum of the group's q>,  v < last   (64 bits, as in select.hip)
//   chosen  = the topk - 1 best of them (ties: the lowest v), and block last;
//   out, lse = softmax attention of the group's G queries over the tokens < L of the
//              chosen blocks.
//
// One launch where few blocks are taken (decode_fused_kernel), else two to four:
// decode_score_kernel scores long tables, decode_select_kernel writes the chosen blocks in ascending
// order, decode_attn_kernel walks them in `parts` runs, decode_merge_kernel puts the
// runs together where there is more than one.
//
// Bound: HBM bytes of the means and of the chosen blocks' keys and values, which are
// read once for the whole group; with few rows the latency of the launches.  Measured:
// 16 sequences of up to 135000 tokens, 8 key heads, 64 blocks of 128: 103 us, 5.6 TB/s in
// all (2 GiB past the caches are read at 7.1); by themselves the selection takes 18 (one
// compute unit a row), the attention 90 and the join 5; 2 x 12 heads, 16 blocks of 64:
// 16 us a call, where what one compute unit reads of its row's 0.5 MB bounds it (twice the
// loads in flight change nothing).

#include <math.h>

#include "attn_tiles.h"
#include "launch.h"
#include "topk_border.h"

namespace sa {

namespace {

constexpr float kLowest = -3.402823466e+38f;

__device__ __forceinline__ int length_of(const DecodeArgs& a, int b) {
  return min(max(a.lengths[b], 0), a.cap);
}

// ---- selection ----
template <int D, int THREADS>
struct ChooseLds {
  double qparts[THREADS / D][D];
  double qsum[D];
  int counts[2][THREADS / 64];
};

// Ordered keys of the scores of blocks v0 .. v1 - 1 of (b, h), to keys[v].  Eight lanes
// take a block's mean, so a wavefront scores eight blocks at a time, two times over to
// have enough loads in flight.  The whole workgroup calls this.
template <int D, int THREADS>
__device__ __forceinline__ void score_blocks(const DecodeArgs& a, int b, int h, int v0, int v1,
                                             uint64_t* keys, ChooseLds<D, THREADS>& lds) {
  const int G = a.Hq / a.Hkv;
  constexpr int P = THREADS / D;  // heads summed side by side
  const int c = threadIdx.x % D, i0 = threadIdx.x / D;
  const __bf16* q = (const __bf16*)a.q + ((int64_t)b * a.Hq + (int64_t)h * G) * D + c;
  double sum = 0.0;
  for (int i = i0; i < G; i += P) sum += (double)(float)q[(int64_t)i * D];
  lds.qparts[i0][c] = sum;
  __syncthreads();
  if (threadIdx.x < D) {
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < P; ++i) sum += lds.qparts[i][c];
    lds.qsum[c] = sum;
  }
  __syncthreads();
  const int part = threadIdx.x & 7;  // columns 4 part + 32 i .. + 3
  double qs[D / 8];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) qs[i] = lds.qsum[4 * part + 32 * (i / 4) + i % 4];
  const float* means = a.means + ((int64_t)b * a.Hkv + h) * a.n_blk * D + 4 * part;
  constexpr int U = 2;  // blocks in flight a lane
  constexpr int kStep = THREADS / 8;
  const int mine = threadIdx.x >> 3;
  for (int w0 = v0; w0 < v1; w0 += U * kStep) {
    f32x4 x[U][D / 32];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        x[u][i] = *(const f32x4*)(means + (int64_t)min(w0 + mine + u * kStep, v1 - 1) * D + 32 * i);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      double t = 0.0;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) t = fma((double)x[u][i / 4][i % 4], qs[i], t);
#pragma unroll
      for (int s = 1; s < 8; s *= 2) t += __shfl_xor(t, s, 64);
      if (part == 0 && w0 + mine + u * kStep < v1) keys[w0 + mine + u * kStep] = order_key(t);
    }
  }
}

// The chosen blocks of a sequence of n blocks, more than topk, from the keys of all but the
// last: in ascending order to `put`'s calls (place, block).  The whole workgroup calls
// this; wavefront 0 writes, so what it puts into LDS needs a barrier.  MOST bounds n.
template <int D, int THREADS, int MOST, typename Put>
__device__ __forceinline__ void choose(int topk, int n, const uint64_t* keys,
                                       ChooseLds<D, THREADS>& lds, Put put) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int last = n - 1;
  const int words = (last + 63) / 64;
  constexpr int kWaves = THREADS / 64;
  constexpr int kEach = MOST / 64 / kWaves;  // words a wavefront of the longest row
  // One wavefront alone where its registers hold the row: a step of all of them takes a
  // barrier (60000 tokens, blocks of 64: 23.7 and 26.4 us a call; 135000: 53.7 with the
  // keys of one wavefront in LDS, 37.9).
  Border edge;
  if (words > 20) {
    if (kEach <= 4 || words <= 4 * kWaves)
      edge = group_border<4, kWaves>(keys, last, topk - 1, wave, lane, lds.counts);
    else
      edge = group_border<kEach <= 4 ? 4 : kEach, kWaves>(keys, last, topk - 1, wave, lane, lds.counts);
  }
  if (wave != 0) return;
  if (words <= 4)
    edge = border_of<4>(keys, last, topk - 1, lane);
  else if (words <= 20)
    edge = border_of<20>(keys, last, topk - 1, lane);
  const uint64_t below = (1ull << lane) - 1ull;
  int done = 0;
  for (int w = 0; w < words; ++w) {
    const uint64_t key = 64 * w + lane < last ? keys[64 * w + lane] : 0;
    uint64_t word = __ballot(key >= edge.lo);
    if (edge.ties >= 0) {
      const uint64_t same = __ballot(key == edge.lo);
      const bool first = key == edge.lo && (int)__popcll(same & below) < edge.ties;
      word = __ballot(key > edge.lo || first);
      edge.ties = max(0, edge.ties - (int)__popcll(same));
    }
    if ((word >> lane) & 1ull) put(done + (int)__popcll(word & below), 64 * w + lane);
    done += __popcll(word);
  }
  if (lane == 0) put(done, last);
}

// Scores of a run of kScoreRun blocks of one (sequence, key head), where a table is long:
// one workgroup a row would read them all through one compute unit.
constexpr int kScoreThreads = 512;
constexpr int kScoreRun = 256;

template <int D>
__global__ __launch_bounds__(kScoreThreads) void decode_score_kernel(DecodeArgs a, int runs) {
  __shared__ ChooseLds<D, kScoreThreads> lds;
  const int bh = blockIdx.x / runs;
  const int b = bh / a.Hkv;
  const int n = (length_of(a, b) + a.blk - 1) / a.blk;
  const int v0 = (int)(blockIdx.x - bh * runs) * kScoreRun, v1 = min(v0 + kScoreRun, n - 1);
  if (n <= a.topk || v0 >= v1) return;
  score_blocks<D, kScoreThreads>(a, b, bh - b * a.Hkv, v0, v1, a.keys + (int64_t)bh * a.n_blk, lds);
}

// A workgroup a (sequence, key head); the scores are its own or decode_score_kernel's.
constexpr int kDecodeSelectThreads = 1024;

template <int D>
__global__ __launch_bounds__(kDecodeSelectThreads) void decode_select_kernel(DecodeArgs a) {
  extern __shared__ uint64_t own_keys[];  // [n_blk], where there are no others
  __shared__ ChooseLds<D, kDecodeSelectThreads> lds;
  const int bh = blockIdx.x;
  const int b = bh / a.Hkv;
  const int n = (length_of(a, b) + a.blk - 1) / a.blk;  // blocks with a token
  int32_t* list = a.blocks + (int64_t)bh * a.topk;
  if (n <= a.topk) {
    // topk may be any int, so i may pass its end
    for (uint32_t i = threadIdx.x; i < (uint32_t)a.topk; i += kDecodeSelectThreads)
      list[i] = (int)i < n ? (int)i : -1;
    return;
  }
  const uint64_t* keys = a.keys + (int64_t)bh * a.n_blk;
  if (!a.keys) {
    score_blocks<D, kDecodeSelectThreads>(a, b, bh - b * a.Hkv, 0, n - 1, own_keys, lds);
    __syncthreads();
    keys = own_keys;
  }
  choose<D, kDecodeSelectThreads, kSelectMaxBlocks>(a.topk, n, keys, lds,
                                                    [&](int at, int v) { list[at] = v; });
}

// ---- attention ----
// D = A B + C for a 16 x 16 fp32 tile with K = 32 bf16: lane l supplies
// A[l % 16][8 (l / 16) + e] and B[8 (l / 16) + e][l % 16], and holds
// C[4 (l / 16) + i][l % 16].
__device__ __forceinline__ f32x4 mfma16x16x32(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Max and sum over lanes l, l ^ 16, l ^ 32 and l ^ 48, by row exchanges in the vector ALU
// (see pair_max).
__device__ __forceinline__ float quad_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

constexpr int kDecodeGroup = 16;  // query heads of a workgroup: one side of an MFMA tile

// A wavefront takes units of 32 keys: S^T = K Q^T with keys straight from memory
// (16 bytes a lane, rows in the order that leaves its probabilities as the second
// product's operand), O^T += V^T P^T with the values through LDS and the transposing
// read.  Keys of the next unit are requested when S is done, its values when this
// unit's are in LDS.  Each wavefront has its own maximum and sums; they meet in LDS.
template <int D, int WAVES>
struct AttendLds {
  __attribute__((aligned(1024))) __bf16 Vs[WAVES][32 * D];
  float stats[WAVES][2][16];
};

// Entries i0 .. i1 - 1 of the list of chosen blocks, block_at(i) for entry i - i0, by the
// workgroup's WAVES wavefronts; part `part` of `parts`.  STREAM: read past the caches.
template <int D, int WAVES, bool STREAM, typename BlockAt>
__device__ __forceinline__ void attend(const DecodeArgs& a, int b, int h, int hg, int part, int parts,
                                       int i0, int i1, BlockAt block_at, AttendLds<D, WAVES>& lds) {
  constexpr int C = D / 8;        // 16-byte chunks of a row
  constexpr int R = 64 / C;       // rows of a load
  constexpr int kVLoads = 32 / R;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int G = a.Hq / a.Hkv;
  const int g0 = hg * kDecodeGroup;
  const int heads = min(kDecodeGroup, G - g0);
  const int len = length_of(a, b);
  const int n = (len + a.blk - 1) / a.blk;
  const int shift = a.blk == 128 ? 2 : 1;  // units of a block: 4 or 2
  const int units = (i1 - i0) << shift;

  bf16x8 qf[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    qf[s] = bf16x8{};
    if (l16 < heads)
      qf[s] = *(const bf16x8*)((const __bf16*)a.q +
                               (((int64_t)b * a.Hq + (int64_t)h * G + g0 + l16) * D + 32 * s + 8 * g));
  }
  const __bf16* K = (const __bf16*)a.k + b * a.sb + h * a.sh;
  const __bf16* V = (const __bf16*)a.v + b * a.sb + h * a.sh;
  const float c_log2 = a.scale * kLog2e;

  auto key0_of = [&](int u) {  // first token of unit u; blocks are below n
    const int blk = min(max(block_at(u >> shift), 0), n - 1);
    return blk * a.blk + ((u & ((1 << shift) - 1)) << 5);
  };
  bf16x8 kf[2][D / 32];
  u32x4 vr[kVLoads];
  auto load = [](const __bf16* p) { return STREAM ? load_stream(p) : *(const u32x4*)p; };
  auto load_k = [&](int key0) {  // rows past the sequence repeat its last one
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const __bf16* row =
          K + (int64_t)min(key0 + 8 * (l16 >> 2) + 4 * t + (l16 & 3), len - 1) * a.sn + 8 * g;
#pragma unroll
      for (int s = 0; s < D / 32; ++s) kf[t][s] = __builtin_bit_cast(bf16x8, load(row + 32 * s));
    }
  };
  auto load_v = [&](int key0) {
#pragma unroll
    for (int i = 0; i < kVLoads; ++i)
      vr[i] = load(V + (int64_t)min(key0 + i * R + lane / C, len - 1) * a.sn + 8 * (lane % C));
  };

  f32x4 o[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i] = f32x4{};
  float m_run = -INFINITY, l_run = 0.f;
  __bf16* vs = lds.Vs[wave];
  int u = wave;
  int key0 = 0;
  if (u < units) {
    key0 = key0_of(u);
    load_k(key0);
    load_v(key0);
  }
  for (; u < units; u += WAVES) {
    f32x4 s2[2] = {};
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) s2[t] = mfma16x16x32(kf[t][s], qf[s], s2[t]);
    const bool more = u + WAVES < units;
    const int key1 = more ? key0_of(u + WAVES) : key0;
    if (more) load_k(key1);
    float x[8];  // key key0 + 8 g + e, query l16
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = key0 + 8 * g + e < len ? s2[e >> 2][e & 3] : -INFINITY;
      mx = fmaxf(mx, x[e]);
    }
    mx = quad_max(mx) * c_log2;
    const float m_new = fmaxf(m_run, mx);
    // a maximum of -inf (nothing seen yet, or logits of -inf only) weighs nothing
    const float m_exp = fmaxf(m_new, kLowest);
    const float alpha = fast_exp2(m_run - m_exp);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] *= alpha;
    // the matrix product takes bf16: a probability is off by 2^-8 of itself there, as in the
    // prompt's attention; the sum adds up the unrounded ones
    bf16x8 pf;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = fast_exp2(fmaf(x[e], c_log2, -m_exp));
      l_run += p;
      pf[e] = (__bf16)p;
    }
#pragma unroll
    for (int i = 0; i < kVLoads; ++i) {
      const int r = i * R + lane / C;
      lds_write_b128(vs + r * D + (((lane % C) ^ swz<D>(r)) << 3), vr[i]);
    }
    if (more) load_v(key1);
    // the wavefront's own writes and reads of LDS complete in order
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int dd = 16 * i + (lane & 3) * 4;
      const int r0 = 8 * g + (l16 >> 2), r1 = r0 + 4;
      const bf16x4 lo = lds_read_tr16_b64(vs + r0 * D + (((dd >> 3) ^ swz<D>(r0)) << 3) + (dd & 7));
      const bf16x4 hi = lds_read_tr16_b64(vs + r1 * D + (((dd >> 3) ^ swz<D>(r1)) << 3) + (dd & 7));
      const bf16x8 vf = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      o[i] = mfma16x16x32(vf, pf, o[i]);
    }
    key0 = key1;
  }
  l_run = quad_sum(l_run);

  // Put the wavefronts together: out = sum_w exp2(m_w - m) O_w over the same sum of l_w.
  float* os = (float*)lds.Vs[0];  // [wave][query][D / 4 chunks, XOR of the query] of 4 floats
  static_assert(sizeof(lds.Vs) >= sizeof(float) * WAVES * 16 * D, "the value tiles hold the sums");
  __syncthreads();
  if (g == 0) {
    lds.stats[wave][0][l16] = m_run;
    lds.stats[wave][1][l16] = l_run;
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {  // o[i][e] is column 16 i + 4 g + e of query l16
    const int ch = (4 * i + g) ^ l16;
    *(SA_LDS f32x4*)(os + (wave * 16 + l16) * D + 4 * ch) = o[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < heads * (D / 4); c += 64 * WAVES) {
    const int qi = c / (D / 4), ch = c % (D / 4);
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, lds.stats[w][0][qi]);
    const float m_exp = fmaxf(m, kLowest);
    float l = 0.f;
    f32x4 t = {};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = fast_exp2(lds.stats[w][0][qi] - m_exp);
      l = fmaf(f, lds.stats[w][1][qi], l);
      t += f * *(const SA_LDS f32x4*)(os + (w * 16 + qi) * D + 4 * (ch ^ qi));
    }
    const int64_t row = (int64_t)b * a.Hq + (int64_t)h * G + g0 + qi;
    if (parts == 1) {
      const float inv = l != 0.f ? 1.0f / l : 0.f;
      *(bf16x4*)((__bf16*)a.out + row * D + 4 * ch) =
          bf16x4{(__bf16)(t[0] * inv), (__bf16)(t[1] * inv), (__bf16)(t[2] * inv), (__bf16)(t[3] * inv)};
      if (ch == 0) a.lse[row] = l != 0.f ? (m + fast_log2(l)) * kLn2 : -INFINITY;
    } else {
      *(f32x4*)(a.parts_out + (row * parts + part) * D + 4 * ch) = t;
      float* ml = a.parts_out + (int64_t)a.B * a.Hq * parts * D + (row * parts + part) * 2;
      if (ch == 0) {
        ml[0] = m;
        ml[1] = l;
      }
    }
  }
}

constexpr int kDecodeWaves = 4;

template <int D, bool STREAM>
__global__ __launch_bounds__(64 * kDecodeWaves) void decode_attn_kernel(DecodeArgs a, int parts,
                                                                        int groups) {
  __shared__ AttendLds<D, kDecodeWaves> lds;
  const int part = blockIdx.x % parts;
  const int rest = blockIdx.x / parts;
  const int bh = rest / groups;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int cnt = min(a.topk, (length_of(a, b) + a.blk - 1) / a.blk);
  const int per = (cnt + parts - 1) / parts;
  const int i0 = min(part * per, cnt), i1 = min(i0 + per, cnt);
  const const_ints list = constant(a.blocks) + (int64_t)bh * a.topk + i0;
  attend<D, kDecodeWaves, STREAM>(a, b, h, rest % groups, part, parts, i0, i1, [&](int i) { return list[i]; },
                          lds);
}

// Selection and attention in one launch, a workgroup a (sequence, key head, group of
// queries), where few blocks are taken: three launches and a join of parts take longer
// than the keys and values themselves.
constexpr int kFusedWaves = 8;
constexpr int kFusedUnits = 64;     // 32 keys each: eight rounds of the wavefronts
constexpr int kFusedBlocks = 2048;  // scores in LDS beside the value tiles

template <int D, bool STREAM>
__global__ __launch_bounds__(64 * kFusedWaves) void decode_fused_kernel(DecodeArgs a, int groups) {
  extern __shared__ uint64_t keys[];  // [n_blk]
  __shared__ AttendLds<D, kFusedWaves> lds;
  __shared__ int32_t list[kFusedUnits / 2];
  static_assert(sizeof(ChooseLds<D, 64 * kFusedWaves>) <= sizeof(lds.Vs), "sums before the values");
  const int bh = blockIdx.x / groups, hg = blockIdx.x % groups;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int blocks = (length_of(a, b) + a.blk - 1) / a.blk;
  const int n = min(blocks, a.topk);
  if (blocks <= a.topk) {
    for (int i = threadIdx.x; i < n; i += 64 * kFusedWaves) list[i] = i;
  } else {
    auto& sums = *(ChooseLds<D, 64 * kFusedWaves>*)lds.Vs;
    score_blocks<D, 64 * kFusedWaves>(a, b, h, 0, blocks - 1, keys, sums);
    __syncthreads();
    choose<D, 64 * kFusedWaves, kFusedBlocks>(a.topk, blocks, keys, sums,
                                              [&](int at, int v) { list[at] = v; });
  }
  __syncthreads();
  if (hg == 0)
    for (int i = threadIdx.x; i < a.topk; i += 64 * kFusedWaves)
      a.blocks[(int64_t)bh * a.topk + i] = i < n ? list[i] : -1;
  attend<D, kFusedWaves, STREAM>(a, b, h, hg, 0, 1, 0, n,
                         [&](int i) { return __builtin_amdgcn_readfirstlane(list[i]); }, lds);
}

// A wavefront a row: its parts' sums, in order.  Lane p holds the weight of part p (64 at a
// time), which the others read from it.
template <int D>
__global__ __launch_bounds__(256) void decode_merge_kernel(DecodeArgs a, int parts) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= (int64_t)a.B * a.Hq) return;
  const float* ml = a.parts_out + (int64_t)a.B * a.Hq * parts * D + row * parts * 2;
  const float* po = a.parts_out + row * parts * D + lane * E;
  float m = -INFINITY, l = 0.f;
  float t[E] = {};
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const int n = min(64, parts - p0);
    float mp = -INFINITY, lp = 0.f;
    if (lane < n) {
      mp = ml[2 * (p0 + lane)];
      lp = ml[2 * (p0 + lane) + 1];
    }
    float top = mp;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s, 64));
    const float m_new = fmaxf(m, top);
    const float m_exp = fmaxf(m_new, kLowest);
    const float keep = fast_exp2(m - m_exp), w = fast_exp2(mp - m_exp);
    m = m_new;
    float sum = w * lp;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s, 64);
    l = fmaf(l, keep, sum);
#pragma unroll
    for (int i = 0; i < E; ++i) t[i] *= keep;
    for (int p = 0; p < n; p += 8) {  // eight parts' sums in flight
      float x[8][E];
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int i = 0; i < E; ++i) x[u][i] = po[(int64_t)(p0 + min(p + u, n - 1)) * D + i];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float f = p + u < n ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), p + u)) : 0.f;
        if (p + u < n)
#pragma unroll
          for (int i = 0; i < E; ++i) t[i] = fmaf(f, x[u][i], t[i]);
      }
    }
  }
  const float inv = l != 0.f ? 1.0f / l : 0.f;
  __bf16* out = (__bf16*)a.out + row * D + lane * E;
#pragma unroll
  for (int i = 0; i < E; ++i) out[i] = (__bf16)(t[i] * inv);
  if (lane == 0) a.lse[row] = l != 0.f ? (m + fast_log2(l)) * kLn2 : -INFINITY;
}

int score_runs(int n_blk) { return (n_blk + kScoreRun - 1) / kScoreRun; }

int head_groups(int Hq, int Hkv) { return (Hq / Hkv + kDecodeGroup - 1) / kDecodeGroup; }

template <int D>
hipError_t launch_d(const DecodeArgs& a, int parts, hipStream_t stream) {
  const int64_t rows = (int64_t)a.B * a.Hkv;
  const int groups = head_groups(a.Hq, a.Hkv);
  const int lds = a.n_blk * 8;
  // chosen keys and values of more than the last cache holds are read past it (16 x 8 rows
  // of 8192 tokens, 537 MB: 117 -> 104 us; 24 rows of 1024, 13 MB: 21.9 and 26.5)
  const bool stream_in =
      rows * (a.topk < a.n_blk ? a.topk : a.n_blk) * a.blk * D * 4 > kLastLevelCache;
  if (parts == 0) {
    hipLaunchKernelGGL((stream_in ? decode_fused_kernel<D, true> : decode_fused_kernel<D, false>),
                       dim3((unsigned)(rows * groups)), dim3(64 * kFusedWaves), lds, stream, a, groups);
    return hipGetLastError();
  }
  if (a.keys) {
    const int runs = score_runs(a.n_blk);
    hipLaunchKernelGGL(decode_score_kernel<D>, dim3((unsigned)(rows * runs)), dim3(kScoreThreads), 0,
                       stream, a, runs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(decode_select_kernel<D>, dim3((unsigned)rows), dim3(kDecodeSelectThreads),
                     a.keys ? 0 : lds, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((stream_in ? decode_attn_kernel<D, true> : decode_attn_kernel<D, false>),
                     dim3((unsigned)(rows * groups * parts)), dim3(64 * kDecodeWaves), 0, stream, a, parts,
                     groups);
  e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  hipLaunchKernelGGL(decode_merge_kernel<D>, dim3((unsigned)(((int64_t)a.B * a.Hq + 3) / 4)),
                     dim3(256), 0, stream, a, parts);
  return hipGetLastError();
}

}  // namespace

// Tables of up to this many blocks are scored where they are chosen from; longer ones in a
// launch of their own, us a call scored in place and apart: 2 rows of 2110 blocks 37.9 and
// 34.4, 1 row of up to 1563 23.6 and 26.3, 128 rows of up to 1055 116.4 and 117.6.
constexpr int kScoredInPlace = 2048;

DecodeWork decode_work(int B, int Hq, int Hkv, int n_blk, int topk, int blk, int d) {
  DecodeWork w{};
  const int64_t rows = (int64_t)B * Hkv * head_groups(Hq, Hkv);
  w.fits = launchable(rows, 64 * kFusedWaves) && launchable((int64_t)B * Hkv, kDecodeSelectThreads);
  if ((int64_t)topk * (blk / 32) <= kFusedUnits && n_blk <= kFusedBlocks) return w;
  // a round of two workgroups a compute unit (16 x 8 rows of 64 blocks: 118.7 us in rounds
  // of half the length, 115.8)
  const int most = topk < n_blk ? topk : n_blk;
  const int64_t parts = (512 + rows - 1) / rows;
  w.parts = (int)(parts < most ? parts : most);
  if (w.parts > 1) w.total = ((size_t)B * Hq * w.parts * (d + 2) * 4 + 255) / 256 * 256;
  w.keys = w.total;
  w.scored = n_blk > kScoredInPlace;
  w.fits = w.fits && launchable(rows * w.parts, 64 * kDecodeWaves) &&
           (!w.scored || launchable((int64_t)B * Hkv * score_runs(n_blk), kScoreThreads));
  if (w.scored) w.total += (size_t)B * Hkv * n_blk * 8;
  return w;
}

hipError_t launch_selected_decode(const DecodeArgs& args, void* workspace, hipStream_t stream) {
  DecodeArgs a = args;
  const DecodeWork w = decode_work(a.B, a.Hq, a.Hkv, a.n_blk, a.topk, a.blk, a.d);
  if (!w.fits) return hipErrorInvalidValue;
  a.parts_out = (float*)workspace;
  a.keys = w.scored ? (uint64_t*)((char*)workspace + w.keys) : nullptr;
  return a.d == 128 ? launch_d<128>(a, w.parts, stream) : launch_d<64>(a, w.parts, stream);
}

}  // namespace sa
