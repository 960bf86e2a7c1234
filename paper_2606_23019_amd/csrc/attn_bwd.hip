// Gradients of block-sparse attention for gfx950.
//
// With P = exp(scale S - lse) over the pairs of the mask, S = Q K^T, and
// D_i = <dout_i, out_i> = sum_j P_ij dP_ij, dP = dO V^T:
//   dV = P^T dO,   dS = P (dP - D),   dQ = scale dS K,   dK = scale dS^T Q.
//
// Two kernels share the work, each without atomics (the same call gives the same
// bits): one walks the key blocks of a query block and sums dQ, one walks the query
// blocks of a key block, by the mask's columns, and sums dK and dV.  Both rebuild S
// and dP, 7 products instead of 5; adding dQ up from the second kernel instead would
// take 64 KB of fp32 atomics for the 21 Mflop of a pair of 128 x 128 blocks, in an
// order that changes from run to run.
//
// Products are v_mfma_f32_32x32x16_bf16 with fp32 accumulators.  A wavefront owns 32
// rows of its item (queries or keys), in registers as the B operand, and its
// accumulators hold the transposed results, so that P and dS come out of the first two
// products as the B operand of the next two (as in the forward kernel): the walked
// tiles are read from LDS by rows for the first and transposed for the second.  P and
// dS are rounded to bf16 there, which the products take.
//
// token_terms makes what both need of a row: lse in the exponent's unit and D, negative,
// so that the accumulators of S and dP can start from them.
//
// Bound: matrix products.  Measured, 12 heads x 32760 tokens (d = 128, blocks of 128,
// density about 0.13): 2.69-2.75 ms, 7 products at 1.10-1.13 PFLOP/s (the forward kernel
// 1.05-1.1; a large library product 1.16-1.35, depending on the card); the 5 that the
// formulas need would take 1.6-1.9 ms at the library's rate.  2 x 10 heads x 4000 tokens
// (d = 64, blocks of 64): 106 us, of which 97-100 in the two kernels at 0.75-0.77 PFLOP/s:
// there compute units are busy for 74 % of the cycles (the start, and an end that the longest
// lists draw out), and while they are, the matrix cores are for 45 % and the vector ALU for
// 42 %, which two wavefronts a SIMD overlap little of.

#include <math.h>

#include <type_traits>

#include "attn_tiles.h"
#include "launch.h"
#include "topk_border.h"

namespace sa {

namespace {

// Workgroup barrier once every wavefront's copies have landed and its reads are done.
__device__ __forceinline__ void barrier_tiles() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A operand, rows of a tile: 32 rows from r0 (in key_of_row order), columns 16 dc ..
template <int D>
__device__ __forceinline__ bf16x8 rows_operand(const __bf16* tile, int r0, int dc, int lane) {
  const int r = r0 + key_of_row(lane & 31);
  return lds_read_b128(tile + r * D + (((2 * dc + (lane >> 5)) ^ swz<D>(r)) << 3));
}

// A operand, a tile transposed: columns 32 dg .. + 31 of rows r0 .. r0 + 15.
template <int D>
__device__ __forceinline__ bf16x8 columns_operand(const __bf16* tile, int r0, int dg, int lane) {
  const int g = lane >> 4, j = lane & 15;
  const int dd = dg * 32 + 16 * (g & 1) + (j & 3) * 4;
  const int ra = r0 + 8 * (g >> 1) + (j >> 2), rb = ra + 4;
  const bf16x4 lo = lds_read_tr16_b64(tile + ra * D + (((dd >> 3) ^ swz<D>(ra)) << 3) + (dd & 7));
  const bf16x4 hi = lds_read_tr16_b64(tile + rb * D + (((dd >> 3) ^ swz<D>(rb)) << 3) + (dd & 7));
  return bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// s += rows of S times b0, p += rows of P times b1(dc), over all columns.  AHEAD requests
// the operands of step dc + 1 before the products of step dc: left to itself the compiler
// reads each just before its use (12 heads x 32760 tokens, d = 128: 2840 -> 2770 us; at d =
// 64 the registers for it are not there, nor for the products by columns at 128).
// A wavefront in these products gives way to one in its exponentials and the products
// after them, which it waits for with more in flight (2740 -> 2670 us; the reverse 2680).
template <int D, bool AHEAD, typename B1>
__device__ __forceinline__ void score_products(f32x16& s, f32x16& p, const __bf16* S, const __bf16* P,
                                               int r0, int lane, const bf16x8 (&b0)[D / 16], B1 b1) {
  if constexpr (!AHEAD) {
#pragma unroll
    for (int dc = 0; dc < D / 16; ++dc) {
      s = mfma32x32x16(rows_operand<D>(S, r0, dc, lane), b0[dc], s);
      p = mfma32x32x16(rows_operand<D>(P, r0, dc, lane), b1(dc), p);
    }
    return;
  }
  bf16x8 x[2], y[2];
  x[0] = rows_operand<D>(S, r0, 0, lane);
  y[0] = rows_operand<D>(P, r0, 0, lane);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int dc = 0; dc < D / 16; ++dc) {
    if (dc + 1 < D / 16) {
      x[(dc + 1) & 1] = rows_operand<D>(S, r0, dc + 1, lane);
      y[(dc + 1) & 1] = rows_operand<D>(P, r0, dc + 1, lane);
    }
    __builtin_amdgcn_sched_barrier(0);
    s = mfma32x32x16(x[dc & 1], b0[dc], s);
    p = mfma32x32x16(y[dc & 1], b1(dc), p);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// ---- lists of the mask's rows and columns ----
// A wavefront each: first the rows (the key blocks of (h, u)), then the columns (the query
// blocks whose row has bit v), both ascending.
__global__ __launch_bounds__(256) void bwd_lists_kernel(BwdArgs a, int row_blocks) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t below = (1ull << lane) - 1ull;
  const int W = (a.n_kb + 63) / 64;
  const int blk = blockIdx.x;
  if (blk < row_blocks) {
    const int64_t row = (int64_t)blk * 4 + wave;
    if (row >= (int64_t)a.mask_heads * a.n_qb) return;
    const uint64_t* words = a.mask + row * W;
    int32_t* list = a.row_lists + row * a.n_kb;
    int done = 0;
    for (int w0 = 0; w0 < W; w0 += 64) {
      // 64 words at a time, handed to the wavefront one by one
      const int real = a.n_kb - (w0 + lane) * 64;
      uint64_t mine = w0 + lane < W ? words[w0 + lane] : 0;
      if (real < 64) mine &= real > 0 ? (1ull << real) - 1ull : 0;
      for (int i = 0; i < min(64, W - w0); ++i) {
        const uint64_t word =
            (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, i) |
            (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), i) << 32;
        if ((word >> lane) & 1ull) list[done + __popcll(word & below)] = (w0 + i) * 64 + lane;
        done += __popcll(word);
      }
    }
    if (lane == 0) a.row_counts[row] = done;
    return;
  }
  const int64_t col = (int64_t)(blk - row_blocks) * 4 + wave;
  if (col >= (int64_t)a.mask_heads * a.n_kb) return;
  const int64_t h = col / a.n_kb;
  const int v = (int)(col - h * a.n_kb);
  const uint64_t* word = a.mask + h * a.n_qb * W + v / 64;
  int32_t* list = a.column_lists + col * a.n_qb;
  int done = 0;
  for (int u0 = 0; u0 < a.n_qb; u0 += 64) {
    const int u = u0 + lane;
    const bool on = u < a.n_qb && ((word[(int64_t)min(u, a.n_qb - 1) * W] >> (v & 63)) & 1ull);
    const uint64_t all = __ballot(on);
    if (on) list[done + __popcll(all & below)] = u;
    done += __popcll(all);
  }
  if (lane == 0) a.column_counts[col] = done;
}

// ---- plan ----
// The workgroups of the two kernels, as tables of (item, first list entry, entries,
// slot).  An item is a query block's or a key block's list.  Columns that every row sees
// are many times longer than the mean, and a short problem has fewer items than the chip
// has places, so
//   - lists of more than `limit` = max(least, total / places) entries are cut into equal
//     parts of at most that, which come first; their sums go to slots of the workspace
//     and bwd_join_kernel adds them up in order;
//   - the others follow in the XCD layout of the forward kernel's schedule (heads in index
//     order), inside every XCD's sequence the longest first by coarse classes, so that
//     long lists do not start last and neighbours still share tiles in L2.
// Places that stay empty have entries < 0.  Measured, 2 x 10 heads x 4000 tokens (d = 64,
// blocks of 64) and 12 x 16000 (64 x 128), us: two classes 127 and 875, four 117 and 822,
// sixteen 120 and 795 (12 x 32760: 2872, 2845, 2816-2880); limits of half the size 12 x
// 8000 224 -> 276.
// Two workgroups of four wavefronts on each of 256 compute units.  Blocks of 64 have three
// or four of two wavefronts there, but their lists are cut no finer.
constexpr int kPlaces = 512;
constexpr int kFront = 2 * kPlaces;     // parts at most: c > limit makes less than c / limit + 1
constexpr int kLeast = 2;               // shortest part, in list entries
constexpr int kStaged = 8192;           // counts that the plan keeps in LDS
constexpr int kSequence = 4096;         // and places of an XCD's sequence
constexpr int kClasses = 4;             // of list length: over 2, 1 and 1 / 2 of the mean, others

struct PlanSide {
  const int32_t* counts;  // [mask_heads][n_own]
  int4* table;            // [front + n_items rounded up to 8]
  int4* splits;           // [kPlaces]: item, first slot, parts
  int32_t* n_splits;
  int n_own, front, n_items, least;
};

// What the two kernels need of a token: rows[bh][n] = {-lse / scale, -D}, past N {-inf, 0} up
// to n_pad.  d / 8 lanes each.
template <int D>
__device__ __forceinline__ void token_terms(const BwdArgs& a, int blk) {
  constexpr int C = D / 8, R = 1024 / C;
  static_assert(128 % R == 0, "n_pad is a multiple of 128");
  const int blocks = a.n_pad / R;
  const int64_t bh = blk / blocks;
  const int n = (blk - (int)bh * blocks) * R + threadIdx.x / C;
  float t = 0.f;
  if (n < a.N) {
    const int64_t at = (bh / a.H) * a.sb + (bh % a.H) * a.sh + (int64_t)n * a.sn + 8 * (threadIdx.x % C);
    const bf16x8 x = *(const bf16x8*)((const __bf16*)a.dout + at);
    const bf16x8 y = *(const bf16x8*)((const __bf16*)a.out + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) t = fmaf((float)x[i], (float)y[i], t);
  }
#pragma unroll
  for (int s = 1; s < C; s *= 2) t += __shfl_xor(t, s, 64);
  if (threadIdx.x % C == 0) {
    a.nlse[bh * a.n_pad + n] = n < a.N ? -a.lse[bh * a.N + n] / a.scale : -INFINITY;
    a.ndelta[bh * a.n_pad + n] = -t;
  }
}

// The plan's workgroups, a sequence or the parts of a side each, and behind them those of the
// tokens' terms, which take longer and hide it.
constexpr int kPlanBlocks = 2 * (kXcds + 1);

template <int D>
__global__ __launch_bounds__(1024) void bwd_plan_kernel(BwdArgs a, PlanSide rows, PlanSide columns,
                                                        int mask_heads, int heads) {
  if (blockIdx.x >= kPlanBlocks) {
    token_terms<D>(a, blockIdx.x - kPlanBlocks);
    return;
  }
  const int place = blockIdx.x % (kXcds + 1);
  __shared__ int sums[1024];
  __shared__ int class_count[kClasses];
  __shared__ int staged[kStaged];  // the counts, where they fit
  __shared__ int seq_item[kSequence];
  __shared__ uint8_t seq_class[kSequence];
  const PlanSide& o = blockIdx.x > kXcds ? columns : rows;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int own = mask_heads * o.n_own;   // counts
  int t = 0;
  for (int i = tid; i < own; i += 1024) {
    const int c = o.counts[i];
    if (own <= kStaged) staged[i] = c;
    t += c;
  }
  const int* counts = own <= kStaged ? staged : o.counts;
  t = wave_sum(t);
  if (lane == 0) sums[wave] = t;
  __syncthreads();
  t = lane < 16 ? sums[lane] : 0;
  t = wave_sum(t);
  __syncthreads();
  const int64_t total = (int64_t)t * (heads / mask_heads);
  const int limit = (int)max((int64_t)o.least, (total + kPlaces - 1) / kPlaces);
  const int mean = max(1, t / own);
  auto count_of = [&](int item) {
    const int bh = item / o.n_own;
    return counts[(int64_t)(bh % mask_heads) * o.n_own + (item - bh * o.n_own)];
  };
  if (place == kXcds) {  // the parts, in the order of the items
    if (o.front == 0) {
      if (tid == 0) *o.n_splits = 0;
      return;
    }
    const int seg = (o.n_items + 1023) / 1024;
    const int i0 = min(tid * seg, o.n_items), i1 = min(i0 + seg, o.n_items);
    int parts = 0, splits = 0;
    for (int i = i0; i < i1; ++i) {
      const int c = count_of(i);
      if (c > limit) {
        parts += (c + limit - 1) / limit;
        ++splits;
      }
    }
    const int mine_sum = parts | splits << 16;  // both at most kFront
    int before = mine_sum;  // inclusive, inside the wavefront
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int x = __shfl_up(before, s, 64);
      before += lane >= s ? x : 0;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < 16; ++w) {
      before += w < wave ? sums[w] : 0;
      all += sums[w];
    }
    before -= mine_sum;
    int slot = before & 0xffff, at = before >> 16;
    for (int i = i0; i < i1; ++i) {
      const int c = count_of(i);
      if (c <= limit) continue;
      const int n = (c + limit - 1) / limit;
      o.splits[at++] = make_int4(i, slot, n, 0);
      for (int p = 0; p < n; ++p, ++slot) {
        const int first = (int)((int64_t)p * c / n);
        o.table[slot] = make_int4(i, first, (int)((int64_t)(p + 1) * c / n) - first, slot);
      }
    }
    const int used = all & 0xffff;
    for (int i = used + tid; i < o.front; i += 1024) o.table[i] = make_int4(0, 0, -1, -1);
    if (tid == 0) *o.n_splits = all >> 16;
    return;
  }
  // sequence x: a wavefront a class, which finds its members' number and then their places
  const int x = place;
  const int units = o.n_items / o.n_own;
  const int len = (o.n_items - x + kXcds - 1) / kXcds;
  int4* seq = o.table + o.front;
  // the item at place j and its class, kClasses if it is cut; all wavefronts work out the
  // first kSequence of them, the divisions of the layout once each
  auto item_at = [&](int j, int* item) {
    int u;
    const int unit = xcd_slice(x + (int64_t)kXcds * j, units, o.n_own, &u);
    *item = unit * o.n_own + u;
    const int c = count_of(*item);
    if (o.front && c > limit) return kClasses;
    return c > 2 * mean ? 0 : c > mean ? 1 : 2 * c > mean ? 2 : 3;
  };
  for (int j = tid; j < min(len, kSequence); j += 1024) {
    int item;
    seq_class[j] = (uint8_t)item_at(j, &item);
    seq_item[j] = item;
  }
  __syncthreads();
  auto mine = [&](int j, int* item) {  // whether place j is of the wavefront's class
    if (j >= len) return false;
    if (j >= kSequence) return item_at(j, item) == wave;
    *item = seq_item[j];
    return seq_class[j] == wave;
  };
  if (wave < kClasses) {
    int item = 0, n = 0;
    for (int j = lane; j < len + lane; j += 64) n += __popcll(__ballot(mine(j, &item)));
    if (lane == 0) class_count[wave] = n;
  }
  __syncthreads();
  int base = 0, all = 0;
  for (int w = 0; w < kClasses; ++w) {
    base += w < wave ? class_count[w] : 0;
    all += class_count[w];
  }
  if (wave < kClasses) {
    for (int j = lane; j < len + lane; j += 64) {
      int item = 0;
      const bool in = mine(j, &item);
      const uint64_t on = __ballot(in);
      if (in)
        seq[x + kXcds * (base + __popcll(on & ((1ull << lane) - 1ull)))] =
            make_int4(item, 0, count_of(item), -1);
      base += __popcll(on);
    }
  }
  for (int j = all + tid; x + kXcds * j < (o.n_items + kXcds - 1) / kXcds * kXcds; j += 1024)
    seq[x + kXcds * j] = make_int4(0, 0, -1, -1);
}

// Rows of a walked tile of the query kernel.  Workgroups of two wavefronts take half at
// d = 128, where that puts three of them on a compute unit instead of two (12 heads x
// 16000 tokens, blocks of 64: 1011 -> 858 us).  At d = 64 whole tiles let four on it, and
// halves of the query side alone, whose LDS is a union with the key side's, no more: 2 x 10
// heads x 4000 tokens, blocks of 64, 106.5 and 110.8 us, 12 x 32760 925 and 948.  Halves of
// both sides make three wavefronts a SIMD of two, for 107.6 and 105.0, 916 and 890, but with
// 128 x 64 blocks 150 and 168 (12 x 8000).
template <int BQ, int D>
constexpr int kWalk = BQ == 64 && D == 128 ? 32 : 64;

// A workgroup's part of an item: `own` block of 32 kWaves rows, its list's entries.
struct Item {
  int64_t bh;
  int block, cnt, slot;
  const_ints list;
};

__device__ __forceinline__ Item item_of(const BwdArgs& a, const BwdSide& l, int place, int n_own,
                                        int n_walked) {
  typedef SA_CONST i32x4* Entries;
  const i32x4 e = *((Entries)(uintptr_t)l.table + place);
  Item r;
  r.bh = e.x / n_own;
  r.block = e.x - (int)r.bh * n_own;
  r.cnt = e.z;
  r.slot = e.w;
  r.list = constant(l.lists) + ((r.bh % a.mask_heads) * n_own + r.block) * n_walked + e.y;
  return r;
}

// Accumulators of a part, as they lie in the registers: 16 floats a lane and column group.
template <int D>
__device__ __forceinline__ void store_part(const f32x16 (&o)[D / 32], float* at, int lane) {
#pragma unroll
  for (int dg = 0; dg < D / 32; ++dg)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *(f32x4*)(at + (dg * 4 + i / 4) * 256 + lane * 4) =
          f32x4{o[dg][i], o[dg][i + 1], o[dg][i + 2], o[dg][i + 3]};
}

// Joins the parts of cut lists: a wavefront 32 rows x 32 columns of one result of one item.
struct JoinSide {
  BwdSide side;
  int n_own, blk, results, blocks;  // results: dQ alone, or dK and dV; blocks of the launch
};

template <int D>
__global__ __launch_bounds__(256) void bwd_join_kernel(BwdArgs a, JoinSide rows, JoinSide columns) {
  const bool first = (int)blockIdx.x < rows.blocks;
  const JoinSide& o = first ? rows : columns;
  const BwdSide& l = o.side;
  const int blk = o.blk, results = o.results, n_own = o.n_own;
  const int per = blk / 32 * (D / 32) * results;  // wavefronts an item
  const int64_t w = (int64_t)(blockIdx.x - (first ? 0 : rows.blocks)) * 4 + (threadIdx.x >> 6);
  const int at = (int)(w / per);
  if (at >= *l.n_splits) return;
  const int4 e = l.splits[at];
  const int unit = (int)(w - (int64_t)at * per);
  const int dg = unit % (D / 32), rest = unit / (D / 32);
  const int which = rest % results, group = rest / results;  // result, 32 rows
  const int lane = threadIdx.x & 63;
  const float* from = l.parts + ((int64_t)e.y * (blk / 32) * results + group * results + which) * (32 * D) +
                      dg * 1024 + lane * 4;
  f32x4 t[4] = {};
  for (int p = 0; p < e.z; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] += *(const f32x4*)(from + (int64_t)p * blk * D * results + i * 256);
  const int64_t bh = e.x / n_own;
  const int row = (e.x - (int)bh * n_own) * blk + group * 32 + (lane & 31);
  if (row >= a.N) return;
  __bf16* out = (__bf16*)(results == 1 ? a.dq : which ? a.dv : a.dk);
  const float f = which ? 1.f : a.scale;
  out += (bh / a.H) * a.sb + (bh % a.H) * a.sh + (int64_t)row * a.sn + dg * 32 + 4 * (lane >> 5);
#pragma unroll
  for (int i = 0; i < 4; ++i) store_out4(out + 8 * i, t[i][0] * f, t[i][1] * f, t[i][2] * f, t[i][3] * f);
}

// ---- dQ ----
template <int BQ, int D>
struct DqLds {
  __attribute__((aligned(1024))) __bf16 tiles[2][2][kWalk<BQ, D> * D];  // buffer, K or V
};

template <int BQ, int D>
__device__ __forceinline__ void bwd_dq(const BwdArgs& a, const BwdSide& side, int place, DqLds<BQ, D>& lds) {
  constexpr int W = kWalk<BQ, D>;
  using T = Tile<BQ, W, D>;
  auto& tiles = lds.tiles;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const Item item = item_of(a, side, place, a.n_qb, a.n_kb);
  if (item.cnt < 0) return;
  const int64_t base = (item.bh / a.H) * a.sb + (item.bh % a.H) * a.sh;
  const __bf16* Kb = (const __bf16*)a.k + base - kCopyShift;
  const __bf16* Vb = (const __bf16*)a.v + base - kCopyShift;
  const int per = a.blk_k / W;  // tiles of a block: 1, 2 or 4
  const int shift = per == 4 ? 2 : per - 1;
  auto block_at = [&](int i) { return min(max(item.list[i], 0), a.n_kb - 1); };
  int n_tiles = 0;
  if (item.cnt > 0) {  // the last block of all may end early
    const int left = min(a.blk_k, a.N - block_at(item.cnt - 1) * a.blk_k);
    n_tiles = ((item.cnt - 1) << shift) + (left + W - 1) / W;
  }
  auto key_of = [&](int t) { return block_at(t >> shift) * a.blk_k + (t & (per - 1)) * W; };
  CopyPlan<T, D> cp;
  cp.init(wave, lane, a.sn);
  auto copy = [&](int t) {
    const int key0 = key_of(t);
    issue_tile_copy<T, W, D>(tiles[t & 1][0], Kb, key0, a.N, a.sn, wave, lane, cp);
    issue_tile_copy<T, W, D>(tiles[t & 1][1], Vb, key0, a.N, a.sn, wave, lane, cp);
  };
  if (n_tiles > 0) copy(0);

  const int row0 = item.block * BQ + wave * 32;
  const int qrow = row0 + l32;
  bf16x8 qf[D / 16], gf[D / 16];
#pragma unroll
  for (int dc = 0; dc < D / 16; ++dc) {
    qf[dc] = gf[dc] = bf16x8{};
    if (qrow < a.N) {
      const int64_t at = base + (int64_t)qrow * a.sn + dc * 16 + half * 8;
      qf[dc] = *(const bf16x8*)((const __bf16*)a.q + at);
      gf[dc] = *(const bf16x8*)((const __bf16*)a.dout + at);
    }
  }
  const float nlse = a.nlse[item.bh * a.n_pad + min(qrow, a.n_pad - 1)];
  const float ndelta = a.ndelta[item.bh * a.n_pad + min(qrow, a.n_pad - 1)];

  f32x16 dq[D / 32];
#pragma unroll
  for (int dg = 0; dg < D / 32; ++dg) dq[dg] = f32x16{};

  for (int t = 0; t < n_tiles; ++t) {
    const __bf16* Ks = tiles[t & 1][0];
    const __bf16* Vs = tiles[t & 1][1];
    const int key0 = key_of(t);
    barrier_tiles();  // tile t landed; every wavefront is done with tile t - 1
    if (t + 1 < n_tiles) copy(t + 1);
#pragma unroll
    for (int kg = 0; kg < W / 32; ++kg) {
      f32x16 s, p;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = nlse;
        p[i] = ndelta;
      }
      __builtin_amdgcn_s_setprio(0);
      score_products<D, D == 128>(s, p, Ks, Vs, kg * 32, lane, qf, [&](int dc) { return gf[dc]; });
      __builtin_amdgcn_s_setprio(1);
      if (key0 + W > a.N) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key0 + kg * 32 + 16 * (i >> 3) + 8 * half + (i & 7) >= a.N) s[i] = -INFINITY;
      }
      bf16x8 ds[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i >> 3][i & 7] = (__bf16)(fast_exp2(s[i] * a.c_log2) * p[i]);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int dg = 0; dg < D / 32; ++dg)
          dq[dg] = mfma32x32x16(columns_operand<D>(Ks, kg * 32 + 16 * c, dg, lane), ds[c], dq[dg]);
    }
  }
  if (item.slot >= 0) {
    store_part<D>(dq, side.parts + ((int64_t)item.slot * (BQ / 32) + wave) * (32 * D), lane);
    return;
  }
  barrier_tiles();  // the tiles are free
  store_rows_staged<D, __bf16>(dq, a.scale, (char*)tiles + wave * (32 * D * 2),
                               (__bf16*)a.dq + base + (int64_t)row0 * a.sn, a.sn, a.N - row0, lane);
}

// ---- dK and dV ----
// The accumulators take 128 registers at d = 128 and the wavefront's K and V rows 64
// more; with S and dP that is past the 256 that let two wavefronts share a SIMD, one's
// exponentials beside the other's MFMAs.  So the V rows stay in LDS there, and to make
// room the walked tiles have 32 rows.
template <int D>
constexpr bool kVInLds = D == 128;
template <int D>
constexpr int kWalkRows = kVInLds<D> ? 32 : 64;

template <int BK, int D>
struct DkvLds {
  __attribute__((aligned(1024))) __bf16 tiles[2][2][kWalkRows<D> * D];  // buffer, Q or dO
  __attribute__((aligned(1024))) __bf16 Vs[kVInLds<D> ? BK * D : 8];
  __attribute__((aligned(1024))) float rows[2][2][64];  // buffer, -lse or -D
};

template <int BK, int D>
__device__ __forceinline__ void bwd_dkv(const BwdArgs& a, const BwdSide& side, int place,
                                        DkvLds<BK, D>& lds) {
  constexpr int W = kWalkRows<D>;
  using T = Tile<BK, W, D>;
  using TV = Tile<BK, BK, D>;
  auto& tiles = lds.tiles;
  auto& Vs = lds.Vs;
  auto& rows = lds.rows;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const Item item = item_of(a, side, place, a.n_kb, a.n_qb);
  if (item.cnt < 0) return;
  const int64_t base = (item.bh / a.H) * a.sb + (item.bh % a.H) * a.sh;
  const __bf16* Qb = (const __bf16*)a.q + base - kCopyShift;
  const __bf16* Gb = (const __bf16*)a.dout + base - kCopyShift;
  const int per = a.blk_q / W;  // tiles of a block: 1, 2 or 4
  const int shift = per == 4 ? 2 : per - 1;
  auto block_at = [&](int i) { return min(max(item.list[i], 0), a.n_qb - 1); };
  int n_tiles = 0;
  if (item.cnt > 0) {  // the last block of all may end early
    const int left = min(a.blk_q, a.N - block_at(item.cnt - 1) * a.blk_q);
    n_tiles = ((item.cnt - 1) << shift) + (left + W - 1) / W;
  }
  auto row_of = [&](int t) { return block_at(t >> shift) * a.blk_q + (t & (per - 1)) * W; };
  CopyPlan<T, D> cp;
  cp.init(wave, lane, a.sn);
  auto copy = [&](int t) {
    const int r0 = row_of(t);
    issue_tile_copy<T, W, D>(tiles[t & 1][0], Qb, r0, a.N, a.sn, wave, lane, cp);
    issue_tile_copy<T, W, D>(tiles[t & 1][1], Gb, r0, a.N, a.sn, wave, lane, cp);
    if (wave < 2) {  // a lane a row, twice where there are 32; all below n_pad
      const float* from = (wave ? a.ndelta : a.nlse) + item.bh * a.n_pad + r0;
      const uint32_t to = __builtin_amdgcn_readfirstlane(
          (uint32_t)(uintptr_t)(SA_LDS void*)rows[t & 1][wave]);
      asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(lane % W * 4), "s"(from), "{m0}"(to)
                   : "memory");
    }
  };
  if constexpr (kVInLds<D>) {
    CopyPlan<TV, D> cv;
    cv.init(wave, lane, a.sn);
    if (n_tiles > 0)
      issue_tile_copy<TV, BK, D>(Vs, (const __bf16*)a.v + base - kCopyShift, item.block * BK, a.N,
                                 a.sn, wave, lane, cv);
  }
  if (n_tiles > 0) copy(0);

  const int row0 = item.block * BK + wave * 32;
  const int krow = min(row0 + l32, a.N - 1);  // rows past N repeat the last: not stored
  bf16x8 kf[D / 16], vf[kVInLds<D> ? 1 : D / 16];
#pragma unroll
  for (int dc = 0; dc < D / 16; ++dc) {
    const int64_t at = base + (int64_t)krow * a.sn + dc * 16 + half * 8;
    kf[dc] = *(const bf16x8*)((const __bf16*)a.k + at);
    if constexpr (!kVInLds<D>) vf[dc] = *(const bf16x8*)((const __bf16*)a.v + at);
  }
  auto v_operand = [&](int dc) {
    if constexpr (!kVInLds<D>) return vf[dc];
    const int r = wave * 32 + l32;
    return lds_read_b128(Vs + r * D + (((2 * dc + half) ^ swz<D>(r)) << 3));
  };
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int dg = 0; dg < D / 32; ++dg) dk[dg] = dv[dg] = f32x16{};

  for (int t = 0; t < n_tiles; ++t) {
    const __bf16* Qs = tiles[t & 1][0];
    const __bf16* Gs = tiles[t & 1][1];
    barrier_tiles();
    if (t + 1 < n_tiles) copy(t + 1);
#pragma unroll
    for (int qg = 0; qg < W / 32; ++qg) {
      f32x16 s, p;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {  // register i holds row 16 (i / 8) + 8 half + i % 8
        const int r = qg * 32 + 16 * (i >> 3) + 8 * half + (i & 7);
        const f32x4 x = *(const SA_LDS f32x4*)(&rows[t & 1][0][r]);
        const f32x4 y = *(const SA_LDS f32x4*)(&rows[t & 1][1][r]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[i + e] = x[e];
          p[i + e] = y[e];
        }
      }
      __builtin_amdgcn_s_setprio(0);
      score_products<D, D == 128>(s, p, Qs, Gs, qg * 32, lane, kf, v_operand);
      __builtin_amdgcn_s_setprio(1);
      bf16x8 pf[2], ds[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = fast_exp2(s[i] * a.c_log2);
        pf[i >> 3][i & 7] = (__bf16)w;
        ds[i >> 3][i & 7] = (__bf16)(w * p[i]);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int dg = 0; dg < D / 32; ++dg) {
          dv[dg] = mfma32x32x16(columns_operand<D>(Gs, qg * 32 + 16 * c, dg, lane), pf[c], dv[dg]);
          dk[dg] = mfma32x32x16(columns_operand<D>(Qs, qg * 32 + 16 * c, dg, lane), ds[c], dk[dg]);
        }
    }
  }
  if (item.slot >= 0) {
    float* at = side.parts + ((int64_t)item.slot * (BK / 32) + wave) * (2 * 32 * D);
    store_part<D>(dk, at, lane);
    store_part<D>(dv, at + 32 * D, lane);
    return;
  }
  barrier_tiles();
  char* slice = (char*)tiles + wave * (32 * D * 2);
  static_assert(sizeof(lds.tiles) >= BK * D * 2, "the tiles hold the results");
  store_rows_staged<D, __bf16>(dk, a.scale, slice, (__bf16*)a.dk + base + (int64_t)row0 * a.sn, a.sn,
                               a.N - row0, lane);
  // the wavefront's own LDS reads and writes complete in order
  store_rows_staged<D, __bf16>(dv, 1.f, slice, (__bf16*)a.dv + base + (int64_t)row0 * a.sn, a.sn,
                               a.N - row0, lane);
}

// Both in one launch where their workgroups are of one size, so that one's last items run
// beside the other's: key blocks first, which take longer.  BQ or BK of 0: the other alone.
template <int BQ, int BK, int D>
union BwdLds {
  DqLds<BQ ? BQ : BK, D> dq;
  DkvLds<BK ? BK : BQ, D> dkv;
};

template <int BQ, int BK, int D>
using LdsOf = std::conditional_t<BQ == 0, DkvLds<BK ? BK : BQ, D>,
                                 std::conditional_t<BK == 0, DqLds<BQ ? BQ : BK, D>, BwdLds<BQ, BK, D>>>;

// Wavefronts on a SIMD that the registers have to leave room for: as many as LDS allows
// workgroups of, up to three at d = 64 and two at 128.  Blocks of 64 at d = 64 have two (34 KB
// of tiles for two wavefronts: four workgroups on a compute unit), dQ alone with blocks of 64
// two or three.
template <int BQ, int BK, int D>
constexpr int kResident = [] {
  constexpr int waves = (BQ ? BQ : BK) / 32, most = D == 64 ? 3 : 2;
  const int by_lds = (160 * 1024 / (int)sizeof(LdsOf<BQ, BK, D>) * waves + 3) / 4;
  return by_lds < most ? by_lds : most;
}();

template <int BQ, int BK, int D>
__global__ __launch_bounds__((BQ ? BQ : BK) * 2, (kResident<BQ, BK, D>)) void bwd_kernel(
    BwdArgs a, BwdSide rows, BwdSide columns, int dkv_places) {
  __shared__ LdsOf<BQ, BK, D> lds;
  if constexpr (BQ == 0) {
    bwd_dkv<BK, D>(a, columns, blockIdx.x, lds);
  } else if constexpr (BK == 0) {
    bwd_dq<BQ, D>(a, rows, blockIdx.x, lds);
  } else {
    if ((int)blockIdx.x < dkv_places)
      bwd_dkv<BK, D>(a, columns, blockIdx.x, lds.dkv);
    else
      bwd_dq<BQ, D>(a, rows, blockIdx.x - dkv_places, lds.dq);
  }
}

// Front entries of a table: parts at most, none where no list can be cut.
int front_of(int64_t items, int n_walked, int least) {
  if (n_walked <= least) return 0;
  const int64_t most = items * ((n_walked + least - 1) / least);
  return (int)(most < kFront ? (most + kXcds - 1) / kXcds * kXcds : kFront);
}

int64_t items_padded(int64_t items) { return (items + kXcds - 1) / kXcds * kXcds; }

// Workgroups of the launches.
struct Grids {
  int64_t row_lists, column_lists, plan, dq, dkv;
};

Grids grids_of(int64_t bh, int64_t mask_heads, int n_qb, int n_kb, int n_pad, int d, const BwdWork& w) {
  return {(mask_heads * n_qb + 3) / 4, (mask_heads * n_kb + 3) / 4,
          kPlanBlocks + bh * (n_pad / (1024 / (d / 8))), w.rows.front + items_padded(bh * n_qb),
          w.columns.front + items_padded(bh * n_kb)};
}

// Every launch reads what the one before it wrote: none goes out behind one that failed.
template <int D>
hipError_t launch_d(const BwdArgs& a, const BwdWork& w, char* ws, hipStream_t stream) {
  const int64_t bh = (int64_t)a.B * a.H;
  const Grids grids = grids_of(bh, a.mask_heads, a.n_qb, a.n_kb, a.n_pad, D, w);
  const int row_blocks = (int)grids.row_lists;
  hipLaunchKernelGGL(bwd_lists_kernel, dim3((unsigned)(grids.row_lists + grids.column_lists)), dim3(256), 0,
                     stream, a, row_blocks);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto side = [&](const BwdSideWork& x, const int32_t* counts, int n_own) {
    return PlanSide{counts, (int4*)(ws + x.table), (int4*)(ws + x.splits), (int32_t*)(ws + x.n_splits),
                    n_own, x.front, (int)(bh * n_own), kLeast};
  };
  const PlanSide rows = side(w.rows, a.row_counts, a.n_qb);
  const PlanSide columns = side(w.columns, a.column_counts, a.n_kb);
  hipLaunchKernelGGL(bwd_plan_kernel<D>, dim3((unsigned)grids.plan), dim3(1024), 0, stream, a, rows,
                     columns, a.mask_heads, (int)bh);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const BwdSide r{a.row_lists, rows.table, rows.splits, rows.n_splits, (float*)(ws + w.rows.parts)};
  const BwdSide c{a.column_lists, columns.table, columns.splits, columns.n_splits,
                  (float*)(ws + w.columns.parts)};
  const int dq_grid = (int)grids.dq, dkv_grid = (int)grids.dkv;
  if (a.blk_q == a.blk_k) {
    const dim3 grid2((unsigned)(dq_grid + dkv_grid));
    if (a.blk_q == 128)
      hipLaunchKernelGGL((bwd_kernel<128, 128, D>), grid2, dim3(256), 0, stream, a, r, c, dkv_grid);
    else
      hipLaunchKernelGGL((bwd_kernel<64, 64, D>), grid2, dim3(128), 0, stream, a, r, c, dkv_grid);
  } else if (a.blk_q == 128) {
    hipLaunchKernelGGL((bwd_kernel<0, 64, D>), dim3(dkv_grid), dim3(128), 0, stream, a, r, c, dkv_grid);
    hipLaunchKernelGGL((bwd_kernel<128, 0, D>), dim3(dq_grid), dim3(256), 0, stream, a, r, c, 0);
  } else {
    hipLaunchKernelGGL((bwd_kernel<0, 128, D>), dim3(dkv_grid), dim3(256), 0, stream, a, r, c, dkv_grid);
    hipLaunchKernelGGL((bwd_kernel<64, 0, D>), dim3(dq_grid), dim3(128), 0, stream, a, r, c, 0);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto join = [&](const BwdSide& x, const PlanSide& p, int blk, int results) {
    const int64_t waves = (int64_t)(p.front / 2) * (blk / 32) * (D / 32) * results;
    return JoinSide{x, p.n_own, blk, results, (int)((waves + 3) / 4)};
  };
  const JoinSide jr = join(r, rows, a.blk_q, 1), jc = join(c, columns, a.blk_k, 2);
  if (jr.blocks + jc.blocks > 0)
    hipLaunchKernelGGL(bwd_join_kernel<D>, dim3((unsigned)(jr.blocks + jc.blocks)), dim3(256), 0, stream,
                       a, jr, jc);
  return hipGetLastError();
}

}  // namespace

BwdWork bwd_work(int B, int H, int mask_heads, int n_qb, int n_kb, int n_pad, int d, int blk_q,
                 int blk_k) {
  BwdWork w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += (bytes + 255) / 256 * 256;
    return from;
  };
  const int64_t bh = (int64_t)B * H;
  auto side = [&](int n_own, int n_walked) {
    BwdSideWork x;
    x.front = front_of(bh * n_own, n_walked, kLeast);
    x.counts = take((size_t)mask_heads * n_own * 4);
    x.lists = take((size_t)mask_heads * n_own * n_walked * 4);
    x.table = take((size_t)(x.front + items_padded(bh * n_own)) * sizeof(int4));
    x.splits = take((size_t)(x.front / 2) * sizeof(int4));
    x.n_splits = take(4);
    return x;
  };
  w.rows = side(n_qb, n_kb);
  w.columns = side(n_kb, n_qb);
  w.nlse = take((size_t)bh * n_pad * 4);
  w.ndelta = take((size_t)bh * n_pad * 4);
  w.rows.parts = take((size_t)w.rows.front * blk_q * d * 4);
  w.columns.parts = take((size_t)w.columns.front * blk_k * d * 8);
  w.total = at;
  const Grids g = grids_of(bh, mask_heads, n_qb, n_kb, n_pad, d, w);
  w.fits = launchable(g.row_lists + g.column_lists, 256) && launchable(g.plan, 1024) &&
           launchable(g.dq + g.dkv, 256);
  return w;
}

hipError_t launch_attention_bwd(const BwdArgs& a, void* workspace, hipStream_t stream) {
  char* ws = (char*)workspace;
  const BwdWork w = bwd_work(a.B, a.H, a.mask_heads, a.n_qb, a.n_kb, a.n_pad, a.d, a.blk_q, a.blk_k);
  if (!w.fits) return hipErrorInvalidValue;
  BwdArgs b = a;
  b.c_log2 = a.scale * kLog2e;
  b.row_counts = (int32_t*)(ws + w.rows.counts);
  b.row_lists = (int32_t*)(ws + w.rows.lists);
  b.column_counts = (int32_t*)(ws + w.columns.counts);
  b.column_lists = (int32_t*)(ws + w.columns.lists);
  b.nlse = (float*)(ws + w.nlse);
  b.ndelta = (float*)(ws + w.ndelta);
  return a.d == 128 ? launch_d<128>(b, w, ws, stream) : launch_d<64>(b, w, ws, stream);
}

}  // namespace sa
