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
// bwd_rows_kernel makes what both need of a row: lse in the exponent's unit and D,
// negative, so that the accumulators of S and dP can start from them.

#include <math.h>

#include "attn_tiles.h"
#include "launch.h"

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

// ---- rows ----
// D / 8 lanes a row.  rows[bh][n] = {-lse / scale, -D}; past N {-inf, 0}, up to n_pad.
template <int D>
__global__ __launch_bounds__(256) void bwd_rows_kernel(BwdArgs a) {
  constexpr int C = D / 8, R = 256 / C;
  const int64_t blocks = (a.n_pad + R - 1) / R;
  const int64_t bh = blockIdx.x / blocks;
  const int n = (int)(blockIdx.x - bh * blocks) * R + threadIdx.x / C;
  if (n >= a.n_pad) return;
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

// ---- lists of a mask's columns ----
// A wavefront a column (h, v): the query blocks whose row has bit v, ascending.
__global__ __launch_bounds__(256) void column_lists_kernel(const uint64_t* __restrict__ mask,
                                                           int64_t columns, int n_qb, int n_kb,
                                                           int32_t* __restrict__ counts,
                                                           int32_t* __restrict__ lists) {
  const int lane = threadIdx.x & 63;
  const int64_t col = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (col >= columns) return;
  const int64_t h = col / n_kb;
  const int v = (int)(col - h * n_kb);
  const int W = (n_kb + 63) / 64;
  const uint64_t* word = mask + h * n_qb * W + v / 64;
  int done = 0;
  for (int u0 = 0; u0 < n_qb; u0 += 64) {
    const int u = u0 + lane;
    const bool on = u < n_qb && ((word[(int64_t)min(u, n_qb - 1) * W] >> (v & 63)) & 1ull);
    const uint64_t all = __ballot(on);
    if (on) lists[col * n_qb + done + __popcll(all & ((1ull << lane) - 1ull))] = u;
    done += __popcll(all);
  }
  if (lane == 0) counts[col] = done;
}

constexpr int kWalk = 64;  // rows of a walked tile

// An item of a kernel's grid: `own` block of 32 kWaves rows and its list of blocks.
struct Item {
  int64_t bh;
  int block;
  const_ints list;
  int cnt;
};

__device__ __forceinline__ Item item_of(const BwdArgs& a, const BwdLists& l, int n_own, int n_walked) {
  const int items = (int)gridDim.x;
  const int it = min(max(constant(l.order)[blockIdx.x], 0), items - 1);
  Item r;
  r.bh = it / n_own;
  r.block = it - (int)r.bh * n_own;
  const int64_t row = (r.bh % a.mask_heads) * n_own + r.block;
  r.cnt = min(max(constant(l.counts)[row], 0), n_walked);
  r.list = constant(l.lists) + row * n_walked;
  return r;
}

// ---- dQ ----
template <int BQ, int D>
__global__ __launch_bounds__(BQ * 2, 2) void bwd_dq_kernel(BwdArgs a, BwdLists lists) {
  using T = Tile<BQ, kWalk, D>;
  __shared__ __attribute__((aligned(1024))) __bf16 tiles[2][2][kWalk * D];  // buffer, K or V
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const Item item = item_of(a, lists, a.n_qb, a.n_kb);
  const int64_t base = (item.bh / a.H) * a.sb + (item.bh % a.H) * a.sh;
  const __bf16* Kb = (const __bf16*)a.k + base - kCopyShift;
  const __bf16* Vb = (const __bf16*)a.v + base - kCopyShift;
  // tiles of kWalk keys: blk_k / kWalk a block, less one where the last block of all ends
  // in its first half
  const int shift = a.blk_k == 128 ? 1 : 0;
  auto block_at = [&](int i) { return min(max(item.list[i], 0), a.n_kb - 1); };
  int n_tiles = item.cnt << shift;
  if (shift && item.cnt > 0 && block_at(item.cnt - 1) * a.blk_k + kWalk >= a.N) --n_tiles;
  auto key_of = [&](int t) { return block_at(t >> shift) * a.blk_k + (shift ? (t & 1) * kWalk : 0); };
  CopyPlan<T, D> cp;
  cp.init(wave, lane, a.sn);
  auto copy = [&](int t) {
    const int key0 = key_of(t);
    issue_tile_copy<T, kWalk, D>(tiles[t & 1][0], Kb, key0, a.N, a.sn, wave, lane, cp);
    issue_tile_copy<T, kWalk, D>(tiles[t & 1][1], Vb, key0, a.N, a.sn, wave, lane, cp);
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
    for (int kg = 0; kg < kWalk / 32; ++kg) {
      f32x16 s, p;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = nlse;
        p[i] = ndelta;
      }
#pragma unroll
      for (int dc = 0; dc < D / 16; ++dc) {
        s = mfma32x32x16(rows_operand<D>(Ks, kg * 32, dc, lane), qf[dc], s);
        p = mfma32x32x16(rows_operand<D>(Vs, kg * 32, dc, lane), gf[dc], p);
      }
      if (key0 + kWalk > a.N) {
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
  barrier_tiles();  // the tiles are free
  store_rows_staged<D, __bf16>(dq, a.scale, (char*)tiles + wave * (32 * D * 2),
                               (__bf16*)a.dq + base + (int64_t)row0 * a.sn, a.sn, a.N - row0, lane);
}

// ---- dK and dV ----
template <int BK, int D>
__global__ __launch_bounds__(BK * 2, 1) void bwd_dkv_kernel(BwdArgs a, BwdLists lists) {
  using T = Tile<BK, kWalk, D>;
  __shared__ __attribute__((aligned(1024))) __bf16 tiles[2][2][kWalk * D];  // buffer, Q or dO
  __shared__ __attribute__((aligned(1024))) float rows[2][2][kWalk];        // buffer, -lse or -D
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const Item item = item_of(a, lists, a.n_kb, a.n_qb);
  const int64_t base = (item.bh / a.H) * a.sb + (item.bh % a.H) * a.sh;
  const __bf16* Qb = (const __bf16*)a.q + base - kCopyShift;
  const __bf16* Gb = (const __bf16*)a.dout + base - kCopyShift;
  const int shift = a.blk_q == 128 ? 1 : 0;
  auto block_at = [&](int i) { return min(max(item.list[i], 0), a.n_qb - 1); };
  int n_tiles = item.cnt << shift;
  if (shift && item.cnt > 0 && block_at(item.cnt - 1) * a.blk_q + kWalk >= a.N) --n_tiles;
  auto row_of = [&](int t) { return block_at(t >> shift) * a.blk_q + (shift ? (t & 1) * kWalk : 0); };
  CopyPlan<T, D> cp;
  cp.init(wave, lane, a.sn);
  auto copy = [&](int t) {
    const int r0 = row_of(t);
    issue_tile_copy<T, kWalk, D>(tiles[t & 1][0], Qb, r0, a.N, a.sn, wave, lane, cp);
    issue_tile_copy<T, kWalk, D>(tiles[t & 1][1], Gb, r0, a.N, a.sn, wave, lane, cp);
    if (wave < 2) {  // r0 + 63 < n_pad
      const float* from = (wave ? a.ndelta : a.nlse) + item.bh * a.n_pad + r0;
      const uint32_t to = __builtin_amdgcn_readfirstlane(
          (uint32_t)(uintptr_t)(SA_LDS void*)rows[t & 1][wave]);
      asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(lane * 4), "s"(from), "{m0}"(to)
                   : "memory");
    }
  };
  if (n_tiles > 0) copy(0);

  const int row0 = item.block * BK + wave * 32;
  const int krow = min(row0 + l32, a.N - 1);  // rows past N repeat the last: not stored
  bf16x8 kf[D / 16], vf[D / 16];
#pragma unroll
  for (int dc = 0; dc < D / 16; ++dc) {
    const int64_t at = base + (int64_t)krow * a.sn + dc * 16 + half * 8;
    kf[dc] = *(const bf16x8*)((const __bf16*)a.k + at);
    vf[dc] = *(const bf16x8*)((const __bf16*)a.v + at);
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int dg = 0; dg < D / 32; ++dg) dk[dg] = dv[dg] = f32x16{};

  for (int t = 0; t < n_tiles; ++t) {
    const __bf16* Qs = tiles[t & 1][0];
    const __bf16* Gs = tiles[t & 1][1];
    barrier_tiles();
    if (t + 1 < n_tiles) copy(t + 1);
#pragma unroll
    for (int qg = 0; qg < kWalk / 32; ++qg) {
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
#pragma unroll
      for (int dc = 0; dc < D / 16; ++dc) {
        s = mfma32x32x16(rows_operand<D>(Qs, qg * 32, dc, lane), kf[dc], s);
        p = mfma32x32x16(rows_operand<D>(Gs, qg * 32, dc, lane), vf[dc], p);
      }
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
  barrier_tiles();
  char* slice = (char*)tiles + wave * (32 * D * 2);
  store_rows_staged<D, __bf16>(dk, a.scale, slice, (__bf16*)a.dk + base + (int64_t)row0 * a.sn, a.sn,
                               a.N - row0, lane);
  // the wavefront's own LDS reads and writes complete in order
  store_rows_staged<D, __bf16>(dv, 1.f, slice, (__bf16*)a.dv + base + (int64_t)row0 * a.sn, a.sn,
                               a.N - row0, lane);
}

template <int D>
hipError_t launch_d(const BwdArgs& a, const BwdLists& rows, const BwdLists& columns,
                    hipStream_t stream) {
  const int64_t bh = (int64_t)a.B * a.H;
  const unsigned dq_grid = (unsigned)(bh * a.n_qb), dkv_grid = (unsigned)(bh * a.n_kb);
  const int R = 256 / (D / 8);
  hipLaunchKernelGGL(bwd_rows_kernel<D>, dim3((unsigned)(bh * ((a.n_pad + R - 1) / R))), dim3(256), 0,
                     stream, a);
  if (a.blk_q == 128)
    hipLaunchKernelGGL((bwd_dq_kernel<128, D>), dim3(dq_grid), dim3(256), 0, stream, a, rows);
  else
    hipLaunchKernelGGL((bwd_dq_kernel<64, D>), dim3(dq_grid), dim3(128), 0, stream, a, rows);
  if (a.blk_k == 128)
    hipLaunchKernelGGL((bwd_dkv_kernel<128, D>), dim3(dkv_grid), dim3(256), 0, stream, a, columns);
  else
    hipLaunchKernelGGL((bwd_dkv_kernel<64, D>), dim3(dkv_grid), dim3(128), 0, stream, a, columns);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_column_lists(const uint64_t* mask_bits, int H, int n_qb, int n_kb, int32_t* counts,
                               int32_t* lists, hipStream_t stream) {
  const int64_t columns = (int64_t)H * n_kb;
  hipLaunchKernelGGL(column_lists_kernel, dim3((unsigned)((columns + 3) / 4)), dim3(256), 0, stream,
                     mask_bits, columns, n_qb, n_kb, counts, lists);
  return hipGetLastError();
}

hipError_t launch_attention_bwd(const BwdArgs& a, const BwdLists& rows, const BwdLists& columns,
                                hipStream_t stream) {
  BwdArgs b = a;
  b.c_log2 = a.scale * kLog2e;
  return a.d == 128 ? launch_d<128>(b, rows, columns, stream) : launch_d<64>(b, rows, columns, stream);
}

}  // namespace sa
