// RMS norm of every head's queries and keys and the rotation by position, in one
// pass, with its gradients.
//
// A row is one token's d elements of one head.  With r = 1 / sqrt(mean x^2 + eps):
//   y = R (x r w),   R turns the first rot elements in pairs: (a, b) ->
//                    (a cos - b sin, a sin + b cos), the rest pass through;
//   n = x r,  g = R^T dy:   dw = sum over rows of g n,
//   dx = r (w g - n mean(w g n)).
//
// Layout: a row is d / 8 lanes of 16 bytes, so a wavefront holds 4 rows (d = 128)
// or 8 (d = 64), those of as many consecutive tokens and one head.  A wavefront
// walks over heads with its tokens fixed: cos, sin and w are loaded once and stay
// in registers, and a store in the [B][H][N][d] layout covers consecutive rows.
// The row sums are DPP steps inside the row's lanes (no LDS).  Pairs of halves
// apart live in two lanes: their raw bf16 values are exchanged (4 dwords).
//
// Bound: HBM bytes (4 an element forward, 6 backward; some 20 vector instructions
// for every 8 elements).  Everything is fp32; each output is rounded to bf16 once.
// Measured: 75600 tokens x 80 heads of 128 in 566 us, 5.5 TB/s (a copy of 2 GiB past the
// caches runs at 6.1); gradients of 2 x 32760 tokens x 24 heads in 224 us, 5.5 TB/s.  Eight
// tokens take 4 us on the GPU and 14 us a call, the host's part.

#include <type_traits>

#include "device_common.h"
#include "launch.h"

namespace sa {

namespace {

constexpr int kRopeWaves = 4;

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}

// Sum over the C lanes (8 or 16, aligned) of a row, in every one of them.
template <int C>
__device__ __forceinline__ float row_sum(float x) {
  x = dpp_add<0xB1>(x);   // lane ^ 1
  x = dpp_add<0x4E>(x);   // lane ^ 2
  x = dpp_add<0x141>(x);  // mirrored inside 8: the other quad, whose lanes are alike
  if constexpr (C == 16) x = dpp_add<0x140>(x);  // mirrored inside 16
  return x;
}

__device__ __forceinline__ void unpack8(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
  return __builtin_bit_cast(u32x4, v);
}

template <bool STREAM>
__device__ __forceinline__ u32x4 load_row(const __bf16* p) {
  if constexpr (STREAM) return load_stream(p);
  return *(const u32x4*)p;
}

// What a lane needs to turn its 8 elements: y = x c + partner s.
template <bool HALVES>
struct Turn {
  float c[HALVES ? 8 : 4], s[HALVES ? 8 : 4];
  int from;  // halves: byte address (4 lane) of the lane that holds the partners

  // chunk: the lane's 16-byte chunk of its row; pos: the row of the tables
  __device__ __forceinline__ void load(const float* cos, const float* sin, int64_t pos, int rot,
                                       int chunk, int lane) {
    constexpr int n = HALVES ? 8 : 4;
    const int half = rot / 2;
    const bool on = 8 * chunk < rot;
    const bool second = HALVES && 8 * chunk >= half;
    const int64_t at = pos * half + (HALVES ? 8 * chunk - (second ? half : 0) : 4 * chunk);
    from = 4 * lane;
    if (HALVES && on) from += second ? -(half / 2) : half / 2;
#pragma unroll
    for (int i = 0; i < n; i += 4) {
      f32x4 cv = {1.f, 1.f, 1.f, 1.f}, sv = {};
      if (on) {
        cv = *(const f32x4*)(cos + at + i);
        sv = *(const f32x4*)(sin + at + i);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[i + e] = cv[e];
        s[i + e] = HALVES && !second ? -sv[e] : sv[e];
      }
    }
  }

  __device__ __forceinline__ u32x4 partners(u32x4 v) const {
    if constexpr (!HALVES) return v;
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)v[i]);
    return p;
  }

  // x turned (SIGN 1) or turned back (-1); p: the partners' elements (halves)
  template <int SIGN>
  __device__ __forceinline__ void apply(float (&x)[8], const float (&p)[8]) const {
    if constexpr (HALVES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaf(p[i], SIGN * s[i], x[i] * c[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = fmaf(b, -SIGN * s[i], a * c[i]);
        x[2 * i + 1] = fmaf(a, SIGN * s[i], b * c[i]);
      }
    }
  }
};

// The lane's tokens: R of them side by side in a wavefront, all B N in one line.
struct Token {
  int64_t b, n, pos;
  bool real;
};

__device__ __forceinline__ Token token_of(const RopeArgs& a, int64_t t) {
  const int64_t total = (int64_t)a.B * a.N;
  Token k;
  k.real = t < total;
  t = k.real ? t : total - 1;
  k.b = t / a.N;
  k.n = t - k.b * a.N;
  k.pos = k.n;
  if (a.positions) k.pos = min(max(a.positions[t], 0), a.n_pos - 1);
  return k;
}

// STREAM: the rows are read past the caches.
template <int D, bool HALVES, bool STREAM>
__global__ __launch_bounds__(64 * kRopeWaves) void norm_rope_kernel(RopeArgs a) {
  constexpr int C = D / 8, R = 64 / C;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = lane % C;
  const int64_t groups = ((int64_t)a.B * a.N + R - 1) / R;
  // a block's wavefronts take neighbouring tokens and the same heads
  const int64_t blocks = (groups + kRopeWaves - 1) / kRopeWaves;
  const int64_t hc = blockIdx.x / blocks;
  const int64_t tg = (blockIdx.x - hc * blocks) * kRopeWaves + wave;
  if (tg >= groups) return;
  const int q_chunks = (a.t[0].H + a.heads - 1) / a.heads;
  const int side = hc < q_chunks ? 0 : 1;
  const RopeSide& o = a.t[side];
  const int h0 = (int)(hc - (side ? q_chunks : 0)) * a.heads;
  const int h1 = min(h0 + a.heads, o.H);

  const Token tok = token_of(a, tg * R + lane / C);
  Turn<HALVES> turn;
  turn.load(a.cos, a.sin, tok.pos, a.rot, chunk, lane);
  float w[8], wp[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[i] = o.w[8 * chunk + i];
    if (HALVES) wp[i] = o.w[8 * (chunk + (turn.from / 4 - lane)) + i];
  }
  const __bf16* x = (const __bf16*)o.x + tok.b * o.sb + tok.n * o.sn + 8 * chunk;
  __bf16* y = (__bf16*)o.y + 8 * chunk;
  int64_t yh;  // elements from head to head
  if (a.bhnd) {
    yh = (int64_t)a.N * D;
    y += tok.b * o.H * yh + tok.n * D;
  } else {
    yh = D;
    y += (tok.b * a.N + tok.n) * o.H * D;
  }
  constexpr int U = 4;  // rows in flight a lane
  for (int h = h0; h < h1; h += U) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_row<STREAM>(x + min(h + u, h1 - 1) * o.sh);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[8], p[8];
      unpack8(v[u], f);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
      const float r = rsqrtf(fmaf(row_sum<C>(ss), 1.0f / D, a.eps));
      if (HALVES) {
        unpack8(turn.partners(v[u]), p);
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] *= r * wp[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= r * w[i];
      turn.template apply<1>(f, p);
      if (tok.real && h + u < h1) {
        if (a.stream_out)
          store_stream(y + (h + u) * yh, pack8(f));
        else
          *(u32x4*)(y + (h + u) * yh) = pack8(f);
      }
    }
  }
}

// Gradients.  A block takes units (token group, run of heads) in a grid-stride loop,
// the queries' first, then the keys', and keeps the lane's 8 columns of dw in
// registers; its sums go to dw_parts[block][side][D], added up by a second kernel in
// a fixed order (no atomics: the same call gives the same bits).
template <int D, bool HALVES, bool STREAM>
__global__ __launch_bounds__(64 * kRopeWaves) void norm_rope_bwd_kernel(RopeArgs a) {
  constexpr int C = D / 8, R = 64 / C;
  __shared__ float sums[kRopeWaves][R][D];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = lane % C;
  const int64_t groups = ((int64_t)a.B * a.N + R - 1) / R;
  const int64_t blocks = (groups + kRopeWaves - 1) / kRopeWaves;
  for (int side = 0; side < 2; ++side) {
    const RopeSide& o = a.t[side];
    const int runs = (o.H + a.heads - 1) / a.heads;
    float w[8], dw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = o.w[8 * chunk + i];
      dw[i] = 0.f;
    }
    for (int64_t unit = blockIdx.x; unit < blocks * runs; unit += gridDim.x) {
      const int64_t hc = unit / blocks;
      const int64_t tg = (unit - hc * blocks) * kRopeWaves + wave;
      if (tg >= groups) continue;
      const int h0 = (int)hc * a.heads;
      const int h1 = min(h0 + a.heads, o.H);
      const Token tok = token_of(a, tg * R + lane / C);
      Turn<HALVES> turn;
      turn.load(a.cos, a.sin, tok.pos, a.rot, chunk, lane);
      const __bf16* x = (const __bf16*)o.x + tok.b * o.sb + tok.n * o.sn + 8 * chunk;
      const __bf16* y = (const __bf16*)o.y + 8 * chunk;
      __bf16* dx = (__bf16*)o.dx + (tok.b * a.N + tok.n) * o.H * D + 8 * chunk;
      int64_t yh;
      if (a.bhnd) {
        yh = (int64_t)a.N * D;
        y += tok.b * o.H * yh + tok.n * D;
      } else {
        yh = D;
        y += (tok.b * a.N + tok.n) * o.H * D;
      }
      constexpr int U = 2;
      for (int h = h0; h < h1; h += U) {
        u32x4 xv[U], yv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          xv[u] = load_row<STREAM>(x + min(h + u, h1 - 1) * o.sh);
          yv[u] = load_row<STREAM>(y + min(h + u, h1 - 1) * yh);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const bool real = tok.real && h + u < h1;
          float f[8], g[8], p[8];
          unpack8(xv[u], f);
          unpack8(yv[u], g);
          if (HALVES) unpack8(turn.partners(yv[u]), p);
          turn.template apply<-1>(g, p);
          float ss = 0.f, along = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            ss = fmaf(f[i], f[i], ss);
            along = fmaf(g[i] * w[i], f[i], along);
          }
          const float r = rsqrtf(fmaf(row_sum<C>(ss), 1.0f / D, a.eps));
          const float m = row_sum<C>(along) * r * (1.0f / D);  // mean of w g n
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float n = f[i] * r;
            dw[i] = fmaf(real ? g[i] : 0.f, n, dw[i]);
            f[i] = r * fmaf(-n, m, g[i] * w[i]);
          }
          if (real) {
            if (a.stream_out)
              store_stream(dx + (int64_t)(h + u) * D, pack8(f));
            else
              *(u32x4*)(dx + (int64_t)(h + u) * D) = pack8(f);
          }
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][lane / C][8 * chunk + i] = dw[i];
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += 64 * kRopeWaves) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < kRopeWaves * R; ++i) t += sums[i / R][i % R][c];
      a.dw_parts[((int64_t)blockIdx.x * 2 + side) * D + c] = t;
    }
  }
}

// dw[side][c]: the blocks' sums, 16 columns a block, in 64 bits.
template <int D>
__global__ __launch_bounds__(256) void norm_rope_dw_kernel(const float* __restrict__ parts, int n,
                                                           float* __restrict__ dwq,
                                                           float* __restrict__ dwk) {
  __shared__ double sums[16][17];
  const int c = blockIdx.x * 16 + threadIdx.x % 16;
  const int row = threadIdx.x / 16;
  double t = 0.0;
#pragma unroll 8
  for (int i = row; i < n; i += 16) t += parts[(int64_t)i * 2 * D + c];
  sums[row][threadIdx.x % 16] = t;
  __syncthreads();
  if (row == 0) {
    t = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += sums[i][threadIdx.x];
    (c < D ? dwq : dwk)[c % D] = (float)t;
  }
}

// Heads a wavefront walks: as many as leave `units` units for the chip (eight wavefronts
// on each SIMD), so that a few tokens still spread over it and many share their tables.
int heads_per_unit(const RopeArgs& a, int64_t units) {
  const int64_t groups = ((int64_t)a.B * a.N + 512 / a.d - 1) / (512 / a.d);
  int heads = 16;
  while (heads > 1 && groups * ((a.t[0].H + heads - 1) / heads + (a.t[1].H + heads - 1) / heads) < units)
    heads /= 2;
  return heads;
}

int64_t rope_blocks(const RopeArgs& a) {
  const int64_t groups = ((int64_t)a.B * a.N + 512 / a.d - 1) / (512 / a.d);
  return (groups + kRopeWaves - 1) / kRopeWaves;
}

// Workgroups of the forward pass, a.heads set.
int64_t forward_grid(const RopeArgs& a) {
  const int64_t runs =
      ((int64_t)a.t[0].H + a.heads - 1) / a.heads + ((int64_t)a.t[1].H + a.heads - 1) / a.heads;
  return rope_blocks(a) * runs;
}

// Results of more than the last cache holds are stored past the caches, rows of more than it
// holds read past it: nothing of them would be left for the next kernel, and they push out
// what is still to be read (75600 tokens x 80 heads: 630 us, 585 with the stores, 566 with
// both).  Below that the next kernel finds them there: with results of 201 MB (32760 x 24)
// stored past the caches the call alone, over and over into the same memory, takes 65 us
// instead of 81, but with the means of its q and k behind it 114 and 110, with the selected
// attention 540 and 533; gradients and a sum of them 188 and 161.
void set_streams(RopeArgs& a, int reads) {
  const int64_t bytes = (int64_t)a.B * a.N * (a.t[0].H + a.t[1].H) * a.d * 2;
  a.stream_out = bytes > kLastLevelCache;
  a.stream_in = reads * bytes > kLastLevelCache;
}

}  // namespace

bool norm_rope_fits(RopeArgs a) {
  a.heads = heads_per_unit(a, 8192);
  return launchable(forward_grid(a), 64 * kRopeWaves);
}

hipError_t launch_norm_rope(RopeArgs a, hipStream_t stream) {
  a.heads = heads_per_unit(a, 8192);
  set_streams(a, 1);
  const int64_t grid = forward_grid(a);
  if (!launchable(grid, 64 * kRopeWaves)) return hipErrorInvalidValue;
  auto pick = [&](auto stream_in) {
    constexpr bool S = decltype(stream_in)::value;
    return a.d == 128 ? (a.halves ? norm_rope_kernel<128, true, S> : norm_rope_kernel<128, false, S>)
                      : (a.halves ? norm_rope_kernel<64, true, S> : norm_rope_kernel<64, false, S>);
  };
  auto kernel = a.stream_in ? pick(std::true_type{}) : pick(std::false_type{});
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kRopeWaves), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_norm_rope_bwd(RopeArgs a, float* dwq, float* dwk, hipStream_t stream) {
  a.heads = heads_per_unit(a, 8192);
  set_streams(a, 2);
  const int64_t runs = (max(a.t[0].H, a.t[1].H) + a.heads - 1) / a.heads;
  const int64_t most = rope_blocks(a) * runs;
  const int grid = (int)(most < kRopeParts ? most : kRopeParts);
  auto pick = [&](auto stream_in) {
    constexpr bool S = decltype(stream_in)::value;
    return a.d == 128
               ? (a.halves ? norm_rope_bwd_kernel<128, true, S> : norm_rope_bwd_kernel<128, false, S>)
               : (a.halves ? norm_rope_bwd_kernel<64, true, S> : norm_rope_bwd_kernel<64, false, S>);
  };
  auto kernel = a.stream_in ? pick(std::true_type{}) : pick(std::false_type{});
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * kRopeWaves), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto add = a.d == 128 ? norm_rope_dw_kernel<128> : norm_rope_dw_kernel<64>;
  hipLaunchKernelGGL(add, dim3(2 * a.d / 16), dim3(256), 0, stream, a.dw_parts, grid, dwq, dwk);
  return hipGetLastError();
}

}  // namespace sa
