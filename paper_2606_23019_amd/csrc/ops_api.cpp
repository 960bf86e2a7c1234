// C ABI of the operators around the attention (declared in include/sa_bsattn.h):
// norm and rotation of q and k, selection of blocks, attention over the selection,
// gradients, single tokens over a cache.  As in api.cpp every argument is checked
// before anything is enqueued.  None of them allocates: workspaces are the caller's.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sa_bsattn.h"
#include "launch.h"

namespace {

constexpr int64_t kMaxInt = ((int64_t)1 << 31) - 1;

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Memory that an argument covers.
struct Span {
  const void* p;
  size_t bytes;
};

inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

// Whether an output shares memory with an input or another output.
template <int NO, int NI>
bool clash(const Span (&outs)[NO], const Span (&ins)[NI]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (overlap(outs[o], ins[i])) return true;
    for (int p = o + 1; p < NO; ++p)
      if (overlap(outs[o], outs[p])) return true;
  }
  return false;
}

// Strides of bf16 rows of d elements: not negative, whole 16 bytes, and no more than
// 2^40 elements from the first row to the end.  n[i] rows are s[i] elements apart.
bool strided(const int64_t* s, const int64_t (&n)[3], int d, size_t* bytes) {
  if (!s) return false;
  int64_t last = d;
  for (int i = 0; i < 3; ++i) {
    if (s[i] < 0 || s[i] % 8 || s[i] > ((int64_t)1 << 40)) return false;
    if (n[i] > 1 && s[i] > ((int64_t)1 << 40) / n[i]) return false;
    last += (n[i] - 1) * s[i];
  }
  *bytes = (size_t)last * 2;
  return true;
}

inline int status(hipError_t e) { return e == hipSuccess ? SA_OK : SA_ERR_HIP; }

inline bool scale_ok(float s) { return s > 0.f && isfinite(s); }

inline bool blk_ok(int b) { return b == 64 || b == 128; }

// ---- norm and rotation ----

// Checks and arguments that both directions share; spans of what both read.
int rope_args(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides,
              const float* wq, const float* wk, const float* cos, const float* sin,
              const int32_t* positions, int B, int N, int Hq, int Hk, int d, int rot, int n_pos,
              float eps, int pairs, int layout, sa::RopeArgs* a, Span (&ins)[7]) {
  if (B < 1 || N < 1 || Hq < 1 || Hk < 1 || n_pos < 1) return SA_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return SA_ERR_UNSUPPORTED;
  if (rot < 16 || rot % 16 || rot > d) return SA_ERR_UNSUPPORTED;
  if (!(eps >= 0.f) || !isfinite(eps)) return SA_ERR_INVALID_ARG;
  if (pairs != SA_PAIRS_INTERLEAVED && pairs != SA_PAIRS_HALVES) return SA_ERR_INVALID_ARG;
  if (layout != SA_LAYOUT_BHND && layout != SA_LAYOUT_BNHD) return SA_ERR_INVALID_ARG;
  if (!positions && n_pos < N) return SA_ERR_INVALID_ARG;
  if (!q || !k || !wq || !wk || !cos || !sin) return SA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(wq, 4) || !aligned(wk, 4) ||
      !aligned(cos, 16) || !aligned(sin, 16) || !aligned(positions, 4))
    return SA_ERR_INVALID_ARG;
  // a token's group and a run of heads are one workgroup's quarter at least
  if ((int64_t)B * N >= ((int64_t)1 << 31) || cdiv((int64_t)B * N, 16) * ((int64_t)Hq + Hk) > kMaxInt)
    return SA_ERR_UNSUPPORTED;
  if (Hq > (1 << 30) || Hk > (1 << 30)) return SA_ERR_UNSUPPORTED;  // a run of heads ends past H
  size_t q_bytes, k_bytes;
  if (!strided(q_strides, {B, N, Hq}, d, &q_bytes) || !strided(k_strides, {B, N, Hk}, d, &k_bytes))
    return SA_ERR_INVALID_ARG;
  const size_t table = (size_t)n_pos * (rot / 2) * 4;
  ins[0] = {q, q_bytes};
  ins[1] = {k, k_bytes};
  ins[2] = {wq, (size_t)d * 4};
  ins[3] = {wk, (size_t)d * 4};
  ins[4] = {cos, table};
  ins[5] = {sin, table};
  ins[6] = {positions, (size_t)B * N * 4};
  *a = sa::RopeArgs{};
  a->t[0] = {q, q_strides[0], q_strides[1], q_strides[2], wq, nullptr, nullptr, Hq};
  a->t[1] = {k, k_strides[0], k_strides[1], k_strides[2], wk, nullptr, nullptr, Hk};
  a->cos = cos;
  a->sin = sin;
  a->positions = positions;
  a->B = B;
  a->N = N;
  a->d = d;
  a->rot = rot;
  a->n_pos = n_pos;
  a->eps = eps;
  a->halves = pairs == SA_PAIRS_HALVES;
  a->bhnd = layout == SA_LAYOUT_BHND;
  return SA_OK;
}

// ---- masks ----

// Bits of a mask argument: shared by the batch entries (1) or one for each (B).
inline bool batches_ok(const void* p, int batches, int B) { return !p || batches == 1 || batches == B; }

int select_shape(int B, int H, int n_qb, int n_kb, int d, int topk) {
  if (B < 1 || H < 1 || n_qb < 1 || n_kb < 1 || topk < 1) return SA_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return SA_ERR_UNSUPPORTED;
  if (n_kb > sa::kSelectMaxBlocks) return SA_ERR_UNSUPPORTED;
  if ((int64_t)B * H * n_qb > kMaxInt || (int64_t)B * H * n_kb > kMaxInt) return SA_ERR_UNSUPPORTED;
  if (!sa::block_select_fits((int64_t)B * H, n_qb, n_kb)) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

// Workspace of sa_selected_attn_fwd: means of q and k, counts, lists, order.
struct SelectedWs {
  size_t qm, km, counts, lists, order, total;
};

SelectedWs selected_ws(int64_t bh, int64_t n_qb, int64_t n_kb, int d) {
  SelectedWs w;
  w.qm = 0;
  w.km = w.qm + align_up((size_t)(bh * n_qb * d) * 4);
  w.counts = w.km + align_up((size_t)(bh * n_kb * d) * 4);
  w.lists = w.counts + align_up((size_t)(bh * n_qb) * 4);
  w.order = w.lists + align_up((size_t)(bh * n_qb * n_kb) * 4);
  w.total = w.order + align_up((size_t)(bh * n_qb) * 4);
  return w;
}

int attn_shape(int B, int H, int N, int d, int blk_q, int blk_k) {
  if (B < 1 || H < 1 || N < 1) return SA_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return SA_ERR_UNSUPPORTED;
  if (!blk_ok(blk_q) || !blk_ok(blk_k)) return SA_ERR_UNSUPPORTED;
  if (cdiv(N, blk_k) > 65535 || cdiv(N, blk_q) > 65535) return SA_ERR_UNSUPPORTED;
  if ((int64_t)B * H * cdiv(N, 8) > kMaxInt) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

int decode_shape(int B, int Hq, int Hkv, int cap, int d, int blk, int topk) {
  if (B < 1 || Hq < 1 || Hkv < 1 || cap < 1 || topk < 1 || Hq % Hkv) return SA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || !blk_ok(blk)) return SA_ERR_UNSUPPORTED;
  if (cdiv(cap, blk) > sa::kSelectMaxBlocks || (int64_t)cap + blk > kMaxInt) return SA_ERR_UNSUPPORTED;
  if ((int64_t)B * Hq * 1024 > kMaxInt) return SA_ERR_UNSUPPORTED;
  if (!sa::decode_work(B, Hq, Hkv, (int)cdiv(cap, blk), topk, blk, d).fits) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

}  // namespace

extern "C" {

SA_API int sa_qk_norm_rope(const void* q, const int64_t* q_strides, const void* k,
                           const int64_t* k_strides, const float* wq, const float* wk,
                           const float* cos, const float* sin, const int32_t* positions,
                           void* q_out, void* k_out, int B, int N, int Hq, int Hk, int d, int rot,
                           int n_pos, float eps, int pairs, int layout, void* stream) {
  sa::RopeArgs a;
  Span ins[7];
  const int st = rope_args(q, q_strides, k, k_strides, wq, wk, cos, sin, positions, B, N, Hq, Hk, d,
                           rot, n_pos, eps, pairs, layout, &a, ins);
  if (st != SA_OK) return st;
  if (!q_out || !k_out || !aligned(q_out, 16) || !aligned(k_out, 16)) return SA_ERR_INVALID_ARG;
  const Span outs[2] = {{q_out, (size_t)B * N * Hq * d * 2}, {k_out, (size_t)B * N * Hk * d * 2}};
  if (clash(outs, ins)) return SA_ERR_INVALID_ARG;
  if (!sa::norm_rope_fits(a)) return SA_ERR_UNSUPPORTED;
  a.t[0].y = q_out;
  a.t[1].y = k_out;
  return status(sa::launch_norm_rope(a, (hipStream_t)stream));
}

SA_API size_t sa_qk_norm_rope_bwd_workspace(int d) {
  return d == 64 || d == 128 ? (size_t)sa::kRopeParts * 2 * d * 4 : 0;
}

SA_API int sa_qk_norm_rope_bwd(const void* dq_out, const void* dk_out, const void* q,
                               const int64_t* q_strides, const void* k, const int64_t* k_strides,
                               const float* wq, const float* wk, const float* cos,
                               const float* sin, const int32_t* positions, void* dq, void* dk,
                               float* dwq, float* dwk, void* workspace, int B, int N, int Hq, int Hk,
                               int d, int rot, int n_pos, float eps, int pairs, int layout,
                               void* stream) {
  sa::RopeArgs a;
  Span both[7];
  const int st = rope_args(q, q_strides, k, k_strides, wq, wk, cos, sin, positions, B, N, Hq, Hk, d,
                           rot, n_pos, eps, pairs, layout, &a, both);
  if (st != SA_OK) return st;
  if (!dq_out || !dk_out || !dq || !dk || !dwq || !dwk || !workspace) return SA_ERR_INVALID_ARG;
  if (!aligned(dq_out, 16) || !aligned(dk_out, 16) || !aligned(dq, 16) || !aligned(dk, 16) ||
      !aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(workspace, 16))
    return SA_ERR_INVALID_ARG;
  const size_t q_bytes = (size_t)B * N * Hq * d * 2, k_bytes = (size_t)B * N * Hk * d * 2;
  const Span ins[9] = {both[0], both[1], both[2], both[3], both[4], both[5], both[6],
                       {dq_out, q_bytes}, {dk_out, k_bytes}};
  const Span outs[5] = {{dq, q_bytes}, {dk, k_bytes}, {dwq, (size_t)d * 4}, {dwk, (size_t)d * 4},
                        {workspace, sa_qk_norm_rope_bwd_workspace(d)}};
  if (clash(outs, ins)) return SA_ERR_INVALID_ARG;
  a.t[0].y = dq_out;
  a.t[1].y = dk_out;
  a.t[0].dx = dq;
  a.t[1].dx = dk;
  a.dw_parts = (float*)workspace;
  return status(sa::launch_norm_rope_bwd(a, dwq, dwk, (hipStream_t)stream));
}

SA_API int sa_block_means(const void* x, const int64_t* x_strides, float* means, int B, int H, int N,
                          int d, int blk, void* stream) {
  if (!x || !means || B < 1 || H < 1 || N < 1) return SA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || !blk_ok(blk)) return SA_ERR_UNSUPPORTED;
  if (!aligned(x, 16) || !aligned(means, 16)) return SA_ERR_INVALID_ARG;
  const int64_t blocks = (int64_t)B * H * cdiv(N, blk);
  if ((int64_t)B * H > kMaxInt || !sa::block_means_fits(blocks) || (int64_t)N + blk > kMaxInt)
    return SA_ERR_UNSUPPORTED;
  size_t bytes;
  if (!strided(x_strides, {B, H, N}, d, &bytes)) return SA_ERR_INVALID_ARG;
  if (overlap({x, bytes}, {means, (size_t)blocks * d * 4})) return SA_ERR_INVALID_ARG;
  return status(sa::launch_block_means({x, x_strides[0], x_strides[1], x_strides[2], means, blk},
                                       {nullptr, 0, 0, 0, nullptr, blk}, B, H, N, d,
                                       (hipStream_t)stream));
}

SA_API int sa_block_select(const float* q_means, const float* k_means, const uint64_t* candidates,
                           int candidate_batches, const uint64_t* keep, int keep_batches,
                           uint64_t* mask_bits, int32_t* counts, int32_t* lists, int B, int H,
                           int n_qb, int n_kb, int d, int topk, void* stream) {
  const int st = select_shape(B, H, n_qb, n_kb, d, topk);
  if (st != SA_OK) return st;
  if (!q_means || !k_means || !mask_bits || !counts != !lists) return SA_ERR_INVALID_ARG;
  if (!batches_ok(candidates, candidate_batches, B) || !batches_ok(keep, keep_batches, B))
    return SA_ERR_INVALID_ARG;
  if (!aligned(q_means, 16) || !aligned(k_means, 16) || !aligned(candidates, 8) || !aligned(keep, 8) ||
      !aligned(mask_bits, 8) || !aligned(counts, 4) || !aligned(lists, 4))
    return SA_ERR_INVALID_ARG;
  const size_t row_words = (size_t)H * n_qb * cdiv(n_kb, 64), rows = (size_t)B * H * n_qb;
  const Span ins[4] = {{q_means, rows * d * 4}, {k_means, (size_t)B * H * n_kb * d * 4},
                       {candidates, row_words * candidate_batches * 8},
                       {keep, row_words * keep_batches * 8}};
  const Span outs[3] = {{mask_bits, row_words * B * 8}, {counts, rows * 4}, {lists, rows * n_kb * 4}};
  if (clash(outs, ins)) return SA_ERR_INVALID_ARG;
  sa::SelectArgs a{q_means, k_means, candidates, keep, mask_bits, counts, lists, nullptr, B, H, n_qb, n_kb, d,
                   topk, candidate_batches > 1, keep_batches > 1};
  return status(sa::launch_block_select(a, (hipStream_t)stream));
}

// The means', the selection's and the attention's launches: the last has up to 2 blk_q
// threads a query block, and some workgroups for the places that stay empty.
static int selected_shape(int B, int H, int N, int d, int blk_q, int blk_k, int topk) {
  int st = attn_shape(B, H, N, d, blk_q, blk_k);
  if (st != SA_OK) return st;
  const int64_t bh = (int64_t)B * H, n_qb = cdiv(N, blk_q), n_kb = cdiv(N, blk_k);
  st = select_shape(B, H, (int)n_qb, (int)n_kb, d, topk);
  if (st != SA_OK) return st;
  if (!sa::block_means_fits(bh * (n_qb + n_kb)) || !sa::launchable(bh * n_qb + 64, 256))
    return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

SA_API size_t sa_selected_attn_workspace(int B, int H, int N, int d, int blk_q, int blk_k) {
  if (selected_shape(B, H, N, d, blk_q, blk_k, 1) != SA_OK) return 0;
  return selected_ws((int64_t)B * H, cdiv(N, blk_q), cdiv(N, blk_k), d).total;
}

SA_API int sa_selected_attn_fwd(const void* q, const void* k, const void* v,
                                const uint64_t* candidates, int candidate_batches,
                                const uint64_t* keep, int keep_batches, void* out, float* lse,
                                uint64_t* mask_bits, void* workspace, int B, int H, int N, int d,
                                int blk_q, int blk_k, int topk, float scale, void* stream) {
  const int st = selected_shape(B, H, N, d, blk_q, blk_k, topk);
  if (st != SA_OK) return st;
  const int n_qb = (int)cdiv(N, blk_q), n_kb = (int)cdiv(N, blk_k);
  if (!q || !k || !v || !out || !lse || !mask_bits || !workspace) return SA_ERR_INVALID_ARG;
  if (!scale_ok(scale)) return SA_ERR_INVALID_ARG;
  if (!batches_ok(candidates, candidate_batches, B) || !batches_ok(keep, keep_batches, B))
    return SA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lse, 4) ||
      !aligned(candidates, 8) || !aligned(keep, 8) || !aligned(mask_bits, 8) || !aligned(workspace, 256))
    return SA_ERR_INVALID_ARG;
  const size_t bytes = (size_t)B * H * N * d * 2;
  const size_t row_words = (size_t)H * n_qb * cdiv(n_kb, 64);
  const SelectedWs w = selected_ws((int64_t)B * H, n_qb, n_kb, d);
  const Span ins[5] = {{q, bytes}, {k, bytes}, {v, bytes},
                       {candidates, row_words * candidate_batches * 8},
                       {keep, row_words * keep_batches * 8}};
  const Span outs[4] = {{out, bytes}, {lse, (size_t)B * H * N * 4}, {mask_bits, row_words * B * 8},
                        {workspace, w.total}};
  if (clash(outs, ins)) return SA_ERR_INVALID_ARG;

  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)workspace;
  float* qm = (float*)(ws + w.qm);
  float* km = (float*)(ws + w.km);
  int32_t* counts = (int32_t*)(ws + w.counts);
  int32_t* lists = (int32_t*)(ws + w.lists);
  int32_t* order = (int32_t*)(ws + w.order);
  const int64_t sb = (int64_t)H * N * d, sh = (int64_t)N * d;
  hipError_t e = sa::launch_block_means({q, sb, sh, d, qm, blk_q}, {k, sb, sh, d, km, blk_k}, B, H, N, d, s);
  // every (batch, head) pair has rows of its own: the attention of B H heads
  const bool reads_mask = sa::attention_reads_mask(1, B * H, n_qb, n_kb, d, blk_q, blk_k);
  if (e == hipSuccess) {
    sa::SelectArgs a{qm, km, candidates, keep, mask_bits, reads_mask ? nullptr : counts,
                     reads_mask ? nullptr : lists, reads_mask ? nullptr : order, B, H, n_qb, n_kb, d,
                     topk, candidate_batches > 1, keep_batches > 1};
    e = sa::launch_block_select(a, s);
  }
  if (e == hipSuccess) {
    sa::AttnArgs a{q, k, v, counts, lists, order, out, lse, 1, B * H, N, d, blk_q, blk_k,
                   n_qb, n_kb, scale, (int64_t)B * H * N * d, sh, d};
    if (reads_mask) a.mask_bits = mask_bits;
    e = sa::launch_attention(a, s);
  }
  return status(e);
}

SA_API size_t sa_bsattn_bwd_workspace(int B, int H, int N, int d, int blk_q, int blk_k,
                                      int mask_batches) {
  if (attn_shape(B, H, N, d, blk_q, blk_k) != SA_OK || (mask_batches != 1 && mask_batches != B)) return 0;
  if ((int64_t)mask_batches * H * cdiv(N, blk_q) > kMaxInt / cdiv(N, blk_k)) return 0;
  const sa::BwdWork w = sa::bwd_work(B, H, mask_batches * H, (int)cdiv(N, blk_q), (int)cdiv(N, blk_k),
                                     (int)(cdiv(N, 128) * 128), d, blk_q, blk_k);
  return w.fits ? w.total : 0;
}

SA_API int sa_bsattn_bwd(const void* dout, const void* q, const void* k, const void* v,
                         const void* out, const float* lse, const uint64_t* mask_bits,
                         int mask_batches, void* dq, void* dk, void* dv, void* workspace, int B,
                         int H, int N, int d, int blk_q, int blk_k, float scale, int layout,
                         void* stream) {
  const int st = attn_shape(B, H, N, d, blk_q, blk_k);
  if (st != SA_OK) return st;
  if (!dout || !q || !k || !v || !out || !lse || !mask_bits || !dq || !dk || !dv || !workspace)
    return SA_ERR_INVALID_ARG;
  // lse / scale has to be a float
  if (!scale_ok(scale) || scale < 1e-30f || (mask_batches != 1 && mask_batches != B))
    return SA_ERR_INVALID_ARG;
  if (layout != SA_LAYOUT_BHND && layout != SA_LAYOUT_BNHD) return SA_ERR_INVALID_ARG;
  const void* rows[8] = {dout, q, k, v, out, dq, dk, dv};
  for (const void* p : rows)
    if (!aligned(p, 16)) return SA_ERR_INVALID_ARG;
  if (!aligned(lse, 4) || !aligned(mask_bits, 8) || !aligned(workspace, 256)) return SA_ERR_INVALID_ARG;
  const bool bnhd = layout == SA_LAYOUT_BNHD;
  // tile copies address a tile with 32-bit byte offsets
  if (bnhd && (int64_t)H * d * 128 * 2 >= ((int64_t)1 << 31)) return SA_ERR_UNSUPPORTED;
  const int n_qb = (int)cdiv(N, blk_q), n_kb = (int)cdiv(N, blk_k);
  const int n_pad = (int)(cdiv(N, 128) * 128);
  const int mask_heads = mask_batches * H;
  if ((int64_t)mask_heads * n_qb > kMaxInt / n_kb) return SA_ERR_UNSUPPORTED;
  const sa::BwdWork work = sa::bwd_work(B, H, mask_heads, n_qb, n_kb, n_pad, d, blk_q, blk_k);
  if (!work.fits) return SA_ERR_UNSUPPORTED;
  const size_t ws_bytes = work.total;
  const size_t bytes = (size_t)B * H * N * d * 2;
  const Span ins[7] = {{dout, bytes}, {q, bytes}, {k, bytes}, {v, bytes}, {out, bytes},
                       {lse, (size_t)B * H * N * 4},
                       {mask_bits, (size_t)mask_heads * n_qb * cdiv(n_kb, 64) * 8}};
  const Span outs[4] = {{dq, bytes}, {dk, bytes}, {dv, bytes}, {workspace, ws_bytes}};
  if (clash(outs, ins)) return SA_ERR_INVALID_ARG;

  sa::BwdArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.dout = dout;
  a.lse = lse;
  a.mask = mask_bits;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.B = B;
  a.H = H;
  a.N = N;
  a.d = d;
  a.blk_q = blk_q;
  a.blk_k = blk_k;
  a.n_qb = n_qb;
  a.n_kb = n_kb;
  a.n_pad = n_pad;
  a.mask_heads = mask_heads;
  a.scale = scale;
  a.sb = (int64_t)H * N * d;
  a.sh = bnhd ? d : (int64_t)N * d;
  a.sn = bnhd ? H * d : d;
  return status(sa::launch_attention_bwd(a, workspace, (hipStream_t)stream));
}

SA_API size_t sa_selected_decode_workspace(int B, int Hq, int Hkv, int cap, int d, int blk, int topk) {
  if (decode_shape(B, Hq, Hkv, cap, d, blk, topk) != SA_OK) return 0;
  return sa::decode_work(B, Hq, Hkv, (int)cdiv(cap, blk), topk, blk, d).total;
}

SA_API int sa_selected_decode(const void* q, const void* k, const void* v, const int64_t* kv_strides,
                              const float* means, const int32_t* lengths, void* out, float* lse,
                              int32_t* blocks, void* workspace, int B, int Hq, int Hkv, int cap,
                              int d, int blk, int topk, float scale, void* stream) {
  const int st = decode_shape(B, Hq, Hkv, cap, d, blk, topk);
  if (st != SA_OK) return st;
  const size_t ws_bytes = sa_selected_decode_workspace(B, Hq, Hkv, cap, d, blk, topk);
  if (!q || !k || !v || !means || !lengths || !out || !lse || !blocks || (ws_bytes && !workspace))
    return SA_ERR_INVALID_ARG;
  if (!scale_ok(scale)) return SA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(means, 16) ||
      !aligned(lengths, 4) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(blocks, 4) ||
      !aligned(workspace, 256))
    return SA_ERR_INVALID_ARG;
  size_t kv_bytes;
  if (!strided(kv_strides, {B, Hkv, cap}, d, &kv_bytes)) return SA_ERR_INVALID_ARG;
  const int n_blk = (int)cdiv(cap, blk);
  const Span ins[5] = {{q, (size_t)B * Hq * d * 2}, {k, kv_bytes}, {v, kv_bytes},
                       {means, (size_t)B * Hkv * n_blk * d * 4}, {lengths, (size_t)B * 4}};
  const Span outs[4] = {{out, (size_t)B * Hq * d * 2}, {lse, (size_t)B * Hq * 4},
                        {blocks, (size_t)B * Hkv * topk * 4},
                        {workspace, ws_bytes}};
  if (clash(outs, ins)) return SA_ERR_INVALID_ARG;
  sa::DecodeArgs a{q, k, v, means, lengths, out, lse, blocks, B, Hq, Hkv, cap, d,
                   blk, n_blk, topk, kv_strides[0], kv_strides[1], kv_strides[2], scale, nullptr, nullptr};
  return status(sa::launch_selected_decode(a, workspace, (hipStream_t)stream));
}

}  // extern "C"
