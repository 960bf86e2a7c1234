// Tiles of the attention kernels in LDS: their swizzle, the asynchronous copies that
// fill them, the barriers between copies and reads, and the store of a wavefront's rows.
#pragma once

#include "device_common.h"

namespace sa {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <int BQ, int BK, int D>
struct Tile {
  static constexpr int kWaves = BQ / 32;
  static constexpr int kThreads = kWaves * 64;
  static constexpr int kChunksPerRow = D / 8;  // 16-byte chunks
  // a tile is copied by wave-wide 1 KB direct-to-LDS loads (64 lanes x 16 B)
  static constexpr int kLoadsPerWave = BK * kChunksPerRow / 64 / kWaves;
  static_assert(BQ % 32 == 0 && BK % 32 == 0 && D % 32 == 0, "tile shape");
  static_assert((BK * kChunksPerRow) % (64 * kWaves) == 0, "copy split");
};

// XOR applied to the 16-byte chunk index of LDS row r (same for K and V
// tiles).  LDS is read 256 bytes (64 banks of 4 bytes) per cycle: 16 lanes of
// a 16-byte read, or 32 lanes of an 8-byte transposing read.
//  d = 128 (a row is one 256-byte bank line, 16 chunks): K operand reads put
//  16 different rows at one logical chunk per cycle -> the XOR must be a
//  bijection on r mod 16; V transposing reads put rows 4k .. 4k + 3 at 4
//  adjacent chunks -> the XORs of those rows must differ in bits 2..3.
//  d = 64 (two rows share a bank line, 8 chunks): the same conditions applied
//  separately to even and odd rows.
template <int D>
__device__ __forceinline__ int swz(int r) {
  static_assert(D == 64 || D == 128, "head dim");
  if constexpr (D == 128)
    return ((r & 3) << 2) | ((r >> 2) & 3);
  else
    return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// Key (within a 32-key group) fed to MFMA row m: bits 2 and 3 of m swapped.
// With this order, register i of the S^T accumulator of lane l holds key
// 16 * (i / 8) + 8 * (l / 32) + (i % 8): eight consecutive keys per half
// wavefront, exactly the B-operand layout of the following P V product.
__device__ __forceinline__ int key_of_row(int m) {
  return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1);
}

// Workgroup barrier after this wave's LDS reads have completed.  Unlike
// __syncthreads() it does not wait for outstanding global->LDS copies.  The
// memory clobber keeps the compiler from moving memory accesses across it.
__device__ __forceinline__ void barrier_lds_reads_done() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Workgroup barrier once all but the VM most recent global->LDS copies of
// every wave have landed (copies complete in issue order).
template <int VM>
__device__ __forceinline__ void barrier_copies_landed() {
  static_assert(VM >= 0 && VM < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(VM) : "memory");
}

// Loads J .. J + COUNT - 1 of a group of four wave-wide direct-to-LDS copies: in
// load j lane l reads 16 bytes at base + off[j] + 1024 j and writes them to LDS
// byte address m0 + 1024 j + 16 l.  Issued as inline assembly so that the
// compiler does not add conservative vmcnt waits before unrelated LDS reads;
// completion is awaited explicitly with barrier_copies_landed().  The
// instruction's offset counts on both sides, so one write of m0 serves a group.
// A direct-to-LDS load needs one wait state after that write, which the compiler
// does not put ahead of inline assembly; with a write and a wait for every load
// masked items of 64 rows were 1-2 % slower (12 heads x 4000 tokens, d = 64,
// density 0.3: 43.5 -> 44.2 us, 41.1 in groups).
template <int J, int COUNT>
__device__ __forceinline__ void copy16_to_lds(uint32_t lds_byte_addr, const void* base,
                                              const uint32_t (&off)[4]) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane(lds_byte_addr);
  if constexpr (COUNT == 4)
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %4 offset:0\n\t"
                 "global_load_lds_dwordx4 %1, %4 offset:1024\n\t"
                 "global_load_lds_dwordx4 %2, %4 offset:2048\n\t"
                 "global_load_lds_dwordx4 %3, %4 offset:%6"
                 ::"v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "{m0}"(m0),
                 "n"(3 * 1024) : "memory");
  else if constexpr (COUNT == 2)
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %2 offset:%4\n\t"
                 "global_load_lds_dwordx4 %1, %2 offset:%5"
                 ::"v"(off[J]), "v"(off[J + 1]), "s"(base), "{m0}"(m0), "n"(1024 * J),
                 "n"(1024 * J + 1024) : "memory");
  else
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:%3"
                 ::"v"(off[J]), "s"(base), "{m0}"(m0), "n"(1024 * J) : "memory");
}

// Per-lane byte offsets of a tile copy.  Lane l of load i writes the 16-byte
// LDS chunk 64 (i + kLoadsPerWave * wave) + l, i.e. row r = R (kLoadsPerWave
// wave + i) + l / C and physical chunk p = l mod C (C chunks per row, R = 64 / C
// rows per load); the XOR swizzle is applied by reading source chunk
// p ^ swz(r).  Source rows are sn elements apart (d for [B][H][N][d] tensors,
// H d for [B][N][H][d]).  The swizzle depends on r mod 16 only, so the lane's
// part of the offset repeats with period 4 in the load index n = kLoadsPerWave
// wave + i, and the rest, R n sn elements, is uniform over the wavefront:
// a plan holds 4 lane offsets, and each load adds its uniform row offset to
// the scalar base address.  (Every real row is congruent mod 16 to the row
// used for its swizzle: R (n - n mod 4) is a multiple of 16.)  The lane offsets
// also hold 1024 (3 - i mod 4), which with the kCopyShift elements that the
// base addresses given to the copies lie below their tensors takes back the
// 1024 (i mod 4) of the load instruction (copy16_to_lds).
constexpr int kCopyShift = 3 * 1024 / 2;
template <typename T, int D>
struct CopyPlan {
  static constexpr int kRowsPerLoad = 64 / T::kChunksPerRow;
  uint32_t lane_off[4];  // byte offset of the lane's chunk for loads with n mod 4 = m
  __device__ __forceinline__ void init(int wave, int lane, int sn) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = (wave * T::kLoadsPerWave + j) & 3;  // n mod 4 of load j, j + 4, ...
      const int lr = lane / T::kChunksPerRow;
      const int p = lane % T::kChunksPerRow;
      const int r = m * kRowsPerLoad + lr;  // row relative to load n - n mod 4
      lane_off[j] = (uint32_t)(r * sn + ((p ^ swz<D>(r)) << 3)) * 2u + 1024u * (3 - j);
    }
  }
  // wavefront-uniform byte offset of load i: rows R (n - n mod 4)
  __device__ __forceinline__ static int64_t row_off(int wave, int i, int sn) {
    const int n = wave * T::kLoadsPerWave + i;
    return (int64_t)((n & ~3) * kRowsPerLoad) * sn * 2;
  }
};

// Whether the loads of a group are issued one by one (one write of m0, but a
// wait each) instead of in one statement.  Masked items of 64 rows at d = 128
// stream the most tile bytes per flop, and where most of those miss in L2 a
// burst of four waits longer than four loads apart: 20 heads x 67609 tokens,
// unstructured masks, density 0.16, in bursts and one by one 11.22 and 10.96 ms
// (10.93 before copies waited for m0), 40 heads at 0.08 11.00 and 10.61 (10.63);
// 32768 tokens 2.68 and 2.69.  Elsewhere bursts are as fast or faster: 128 x 128
// 0.1-1 %.
template <typename T, int D>
constexpr bool kCopySpread = T::kWaves == 2 && D == 128;

// Loads i0 .. i0 + count - 1 of a copy of rows key0 .. key0 + BK - 1 (rows sn
// elements apart, row 0 at src + kCopyShift) into an LDS tile with global_load_lds_dwordx4 (no
// registers; completion is tracked by vmcnt).  count and i0 are compile-time
// constants wherever this is inlined into an unrolled loop.  In a ragged last
// block, rows past N repeat row N - 1: finite values whose logits are masked
// and whose probabilities are exactly zero.
template <typename T, int BK, int D>
__device__ __forceinline__ void issue_tile_slice(__bf16* lds, const __bf16* src, int key0, int N,
                                                 int sn, int wave_u, int lane,
                                                 const CopyPlan<T, D>& cp, int i0, int count) {
  const char* tile = (const char*)(src + (int64_t)key0 * sn);
  const uint32_t lds0 =
      (uint32_t)(uintptr_t)(SA_LDS void*)lds + (uint32_t)(wave_u * T::kLoadsPerWave * 1024);
  if (key0 + BK <= N) {
    const int step = count % 4 ? 2 : 4;  // slices begin at a multiple of their group's length
#pragma unroll
    for (int i = i0; i < i0 + count; i += step) {
      const char* from = tile + CopyPlan<T, D>::row_off(wave_u, i, sn);
      if (step == 4 && kCopySpread<T, D>) {
        copy16_to_lds<0, 1>(lds0 + i * 1024, from, cp.lane_off);
        copy16_to_lds<1, 1>(lds0 + i * 1024, from, cp.lane_off);
        copy16_to_lds<2, 1>(lds0 + i * 1024, from, cp.lane_off);
        copy16_to_lds<3, 1>(lds0 + i * 1024, from, cp.lane_off);
      } else if (step == 4)
        copy16_to_lds<0, 4>(lds0 + i * 1024, from, cp.lane_off);
      else if ((i & 3) == 0)
        copy16_to_lds<0, 2>(lds0 + i * 1024, from, cp.lane_off);
      else
        copy16_to_lds<2, 2>(lds0 + (i & ~3) * 1024, from, cp.lane_off);
    }
  } else {
    // Row R n + lr of the tile is read from row min(R n + lr, last), addressed
    // from the tile start: lane_off covers rows R (n mod 4) + lr, so the rows
    // still to add are min(R (n - n mod 4), last - R (n mod 4) - lr), which is
    // negative when the clamped row lies below row R (n - n mod 4).  The sum
    // is taken mod 2^32 and equals the true offset, which is non-negative and
    // inside the tile.  (Adding a negative row count to the uniform base of a
    // full-tile load instead would wrap the 32-bit lane offset.)
    const int last = N - 1 - key0;  // last real row of this tile
    int lr = lane / T::kChunksPerRow;
    // opaque to the optimiser: keeps the per-load row sums below from being
    // hoisted out of the block loop, where they would hold 4 registers
    asm volatile("" : "+v"(lr));
#pragma unroll
    for (int i = i0; i < i0 + count; ++i) {
      const int n = wave_u * T::kLoadsPerWave + i;
      constexpr int R = CopyPlan<T, D>::kRowsPerLoad;
      const int rows = min((n & ~3) * R, last - (n & 3) * R - lr);
      uint32_t off[4];
      off[i & 3] = cp.lane_off[i & 3] + (uint32_t)(rows * sn) * 2u;
      const uint32_t to = lds0 + (i & ~3) * 1024;
      switch (i & 3) {
        case 0: copy16_to_lds<0, 1>(to, tile, off); break;
        case 1: copy16_to_lds<1, 1>(to, tile, off); break;
        case 2: copy16_to_lds<2, 1>(to, tile, off); break;
        default: copy16_to_lds<3, 1>(to, tile, off);
      }
    }
  }
}

// A whole tile copy.
template <typename T, int BK, int D>
__device__ __forceinline__ void issue_tile_copy(__bf16* lds, const __bf16* src, int key0, int N,
                                                int sn, int wave_u, int lane,
                                                const CopyPlan<T, D>& cp) {
  issue_tile_slice<T, BK, D>(lds, src, key0, N, sn, wave_u, lane, cp, 0, T::kLoadsPerWave);
}

// Four consecutive outputs of a row: bf16 (round to nearest even) or fp32.
__device__ __forceinline__ void store_out4(__bf16* p, float a, float b, float c, float d) {
  *(bf16x4*)p = bf16x4{(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
}
__device__ __forceinline__ void store_out4(float* p, float a, float b, float c, float d) {
  *(f32x4*)p = f32x4{a, b, c, d};
}

// Output epilogue through LDS.  In the accumulator layout lane l holds 64
// values of query row l mod 32, so a direct store instruction writes 16
// bytes into each of 32 rows.  Here the wavefront's 32 rows, normalised and
// converted, go into a free LDS slice in row-major order (16-byte chunk c of
// row r at chunk c ^ (r mod C), C chunks per row, conflict-free both ways)
// and are read back so that each lane stores 16 contiguous bytes and a store
// instruction covers whole rows.  The slice is this wavefront's own and
// wavefront-local LDS accesses complete in order, so no barrier is needed.
// out0 is row 0 of the wavefront's rows (rows sn elements apart); rows at or
// past n_rows are not stored.
template <int D, typename OutT>
__device__ __forceinline__ void store_rows_staged(const f32x16 (&o)[D / 32], float inv,
                                                  char* slice, OutT* out0, int sn, int n_rows,
                                                  int lane) {
  constexpr int kChunk = 16 / (int)sizeof(OutT);  // elements per 16-byte chunk
  constexpr int C = D / kChunk;                   // chunks per row
  constexpr int kRowBytes = D * (int)sizeof(OutT);
  const int r = lane & 31;
  const int half = lane >> 5;
#pragma unroll
  for (int dg = 0; dg < D / 32; ++dg)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      // elements d = 32 dg + 8 r4 + 4 half + 0..3 of row r
      const float a = o[dg][4 * r4 + 0] * inv, b = o[dg][4 * r4 + 1] * inv;
      const float c = o[dg][4 * r4 + 2] * inv, d = o[dg][4 * r4 + 3] * inv;
      if constexpr (sizeof(OutT) == 2) {
        const int ch = 4 * dg + r4;
        *(SA_LDS bf16x4*)(slice + r * kRowBytes + ((ch ^ (r % C)) << 4) + 8 * half) =
            bf16x4{(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
      } else {
        const int ch = 8 * dg + 2 * r4 + half;
        *(SA_LDS f32x4*)(slice + r * kRowBytes + ((ch ^ (r % C)) << 4)) = f32x4{a, b, c, d};
      }
    }
  constexpr int kRowsPerStore = 64 / C;
  constexpr int kStores = 32 / kRowsPerStore;
  const int cl = lane % C;
  const int rl = lane / C;
  // All read-backs go out before the first store: the empty asm takes each
  // value where it is read, so the reads are not sunk into the guarded
  // stores below, where each would wait for its own LDS round trip.
  u32x4 v[kStores];
#pragma unroll
  for (int j = 0; j < kStores; ++j) {
    const int row = j * kRowsPerStore + rl;
    v[j] = *(const SA_LDS u32x4*)(slice + row * kRowBytes + ((cl ^ (row % C)) << 4));
  }
#pragma unroll
  for (int j = 0; j < kStores; ++j) asm volatile("" : "+v"(v[j]));
#pragma unroll
  for (int j = 0; j < kStores; ++j) {
    const int row = j * kRowsPerStore + rl;
    if (row < n_rows) *(u32x4*)(out0 + ((uint32_t)(row * sn) + (uint32_t)(cl * kChunk))) = v[j];
  }
}

}  // namespace

}  // namespace sa
