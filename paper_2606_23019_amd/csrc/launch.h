// Internal host-side launchers shared by the C ABI (api.cpp) and the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sa {

// Largest B * H for which the schedule sorts (b, h) groups by cost; larger
// problems keep the natural item order.
constexpr int kScheduleMaxUnits = 4096;

// Whether HIP takes a launch of so many workgroups: fewer than 2^32 threads in all.
constexpr bool launchable(int64_t workgroups, int threads) {
  return workgroups <= (((int64_t)1 << 32) - 1) / threads;
}

// Bytes of the last cache before HBM.
constexpr int64_t kLastLevelCache = 256 << 20;

struct AttnArgs {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* counts;
  const int32_t* lists;
  const int32_t* order;
  void* out;
  float* lse;
  int B, H, N, d, blk_q, blk_k, n_qb, n_kb;
  float scale;
  // element strides of q, k, v and out: batch, head, token (the head-dim is contiguous)
  int64_t sb, sh;
  int sn;
  bool out_f32 = false;  // out is fp32 instead of bf16 (masked path only)
  // mask rows, in place of counts, lists and order, where attention_reads_mask()
  const uint64_t* mask_bits = nullptr;
};

// One side (queries or keys) of the norm and rotation: x with element strides of
// batch, token and head (the head-dim is contiguous), y or its gradient in the
// output's layout, dx contiguous [B][N][H][d].
struct RopeSide {
  const void* x;
  int64_t sb, sn, sh;
  const float* w;
  const void* y;
  void* dx;
  int H;
};

struct RopeArgs {
  RopeSide t[2];
  const float* cos;
  const float* sin;
  const int32_t* positions;
  float* dw_parts;  // gradients only: float [kRopeParts][2][d]
  int B, N, d, rot, n_pos;
  float eps;
  bool halves, bhnd;
  // set by the launchers
  int heads;
  bool stream_in, stream_out;
};

// Blocks of the gradients' kernel at most, each with its own sums for dw.
constexpr int kRopeParts = 1024;

// Whether the forward pass of this size can be launched (the gradients' always can).
bool norm_rope_fits(RopeArgs a);

hipError_t launch_norm_rope(RopeArgs a, hipStream_t stream);
hipError_t launch_norm_rope_bwd(RopeArgs a, float* dwq, float* dwk, hipStream_t stream);

// Block means of one tensor, or of two: x (null: none) with element strides of batch, head
// and token.
struct MeansArgs {
  const void* x;
  int64_t sb, sh, sn;
  float* means;
  int blk;
};

// `blocks`: of one tensor, or of both.
bool block_means_fits(int64_t blocks);

hipError_t launch_block_means(const MeansArgs& q, const MeansArgs& k, int B, int H, int N, int d,
                              hipStream_t stream);

// Most key blocks of a row that is selected: its keys have to fit in LDS.
constexpr int kSelectMaxBlocks = 16384;

struct SelectArgs {
  const float* qm;
  const float* km;
  const uint64_t* candidates;  // or null
  const uint64_t* keep;        // or null
  uint64_t* bits;
  int32_t* counts;  // with lists, or both null
  int32_t* lists;
  int32_t* order;   // the attention kernel's order of B H heads' items, or null
  int B, H, n_qb, n_kb, d, topk;
  bool cand_per_batch, keep_per_batch;
};

bool block_select_fits(int64_t heads, int n_qb, int n_kb);

hipError_t launch_block_select(const SelectArgs& a, hipStream_t stream);

// Single-token attention over selected blocks of a cache.
struct DecodeArgs {
  const void* q;
  const void* k;
  const void* v;
  const float* means;
  const int32_t* lengths;
  void* out;
  float* lse;
  int32_t* blocks;
  int B, Hq, Hkv, cap, d, blk, n_blk, topk;
  int64_t sb, sh, sn;  // element strides of k and v: batch, head, token
  float scale;
  // set by the launcher
  float* parts_out;  // parts > 1: float [B][Hq][parts][d], then [B][Hq][parts][2]
  uint64_t* keys;    // scores of long tables [B][Hkv][n_blk], or null
};

// Parts that a row's blocks are walked in, each by a workgroup of its own (0: selection and
// attention are one launch), and the workspace: their sums, then the scores if `scored`.
struct DecodeWork {
  int parts;
  bool scored;
  bool fits;  // the launches are of sizes that HIP takes
  size_t keys, total;
};

DecodeWork decode_work(int B, int Hq, int Hkv, int n_blk, int topk, int blk, int d);

hipError_t launch_selected_decode(const DecodeArgs& a, void* workspace, hipStream_t stream);

struct BwdArgs {
  const void* q;
  const void* k;
  const void* v;
  const void* out;
  const void* dout;
  const float* lse;
  const uint64_t* mask;
  void* dq;
  void* dk;
  void* dv;
  int B, H, N, d, blk_q, blk_k, n_qb, n_kb;
  int n_pad;       // N rounded up to 128
  int mask_heads;  // H, or B H with a mask for every batch entry
  float scale;
  int64_t sb, sh;  // element strides: batch, head, token
  int sn;
  // set by the launcher: the exponent's factor, and the workspace
  float c_log2;
  int32_t* row_counts;     // [mask_heads][n_qb]
  int32_t* row_lists;      // [mask_heads][n_qb][n_kb]
  int32_t* column_counts;  // [mask_heads][n_kb]
  int32_t* column_lists;   // [mask_heads][n_kb][n_qb]
  float* nlse;             // [B H][n_pad]
  float* ndelta;
};

// Lists that a kernel walks, and the plan of its workgroups.
struct BwdSide {
  const int32_t* lists;
  const int4* table;
  const int4* splits;
  const int32_t* n_splits;
  float* parts;  // sums of the parts, a slot each
};

// Offsets in the workspace; `front`: entries of a table for parts of cut lists.
struct BwdSideWork {
  size_t counts, lists, table, splits, n_splits, parts;
  int front;
};

struct BwdWork {
  BwdSideWork rows, columns;
  size_t nlse, ndelta, total;
  bool fits;  // the launches are of sizes that HIP takes
};

BwdWork bwd_work(int B, int H, int mask_heads, int n_qb, int n_kb, int n_pad, int d, int blk_q,
                 int blk_k);

hipError_t launch_attention_bwd(const BwdArgs& a, void* workspace, hipStream_t stream);

hipError_t launch_prepass(const uint64_t* mask_bits, int H, int n_qb, int n_kb, int32_t* counts,
                          int32_t* lists, hipStream_t stream);

hipError_t launch_schedule(const int32_t* counts, int B, int H, int n_qb, int32_t* order,
                           hipStream_t stream);

hipError_t launch_mask_instantiate(const float* T, const float* p, int n_p, int H, int n_qb,
                                   int n_kb, uint64_t* bits, hipStream_t stream);

hipError_t launch_resize_map(const float* T, int H, int nq, int nk, float* out, int tq, int tk,
                             hipStream_t stream);

hipError_t launch_resize_mask(const uint64_t* bits, int H, int nq, int nk, uint64_t* out, int tq,
                              int tk, hipStream_t stream);

bool fidelity_supported(int R, int K);

hipError_t launch_fidelity(const void* q, const void* k, const int32_t* rows, int R, const float* T,
                           const float* p, int K, float* blk_lse, float* hel, float* fid, int B,
                           int H, int N, int d, int blk, float scale, hipStream_t stream);

// Whether the attention kernel of this shape can walk the mask rows itself.
bool attention_reads_mask(int B, int H, int n_qb, int n_kb, int d, int blk_q, int blk_k);

hipError_t launch_attention(const AttnArgs& a, hipStream_t stream);

// Maskless variant: every key block enabled; counts, lists and order unused.
hipError_t launch_attention_dense(const AttnArgs& a, hipStream_t stream);

}  // namespace sa
