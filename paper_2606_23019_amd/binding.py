"""ctypes binding of ``libsa_bsattn.so`` (C ABI declared in include/sa_bsattn.h).

Argument marshalling only: every step of the forward pass runs in the HIP
library.  PyTorch supplies device buffers and the current stream.  There is no
fallback: if the library cannot be loaded the functions raise.
"""

import ctypes
import functools
import os

import numpy as np

from . import build as _build

SA_OK = 0
SA_ERR_INVALID_ARG = 1
SA_ERR_UNSUPPORTED = 2
SA_ERR_HIP = 3
SA_ERR_TOO_LARGE = 4
SA_LAYOUT_BHND = 0
SA_LAYOUT_BNHD = 1
SA_PAIRS_INTERLEAVED = 0
SA_PAIRS_HALVES = 1

_LIB = None

_P = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float
_Z = ctypes.c_size_t
_S = ctypes.POINTER(ctypes.c_int64)  # element strides

# name -> (restype, argtypes); mirrors include/sa_bsattn.h
SIGNATURES = {
    "sa_status_string": (ctypes.c_char_p, [_I]),
    "sa_version": (_I, []),
    "sa_bsattn_fwd": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P]),
    "sa_mask_prepass": (_I, [_P, _I, _I, _I, _P, _P, _P]),
    "sa_schedule": (_I, [_P, _I, _I, _I, _P, _P]),
    "sa_bsattn_fwd_prepared": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P]),
    "sa_bsattn_plan_create": (_I, [_P, _I, _I, _I, _I, _I, _P, ctypes.POINTER(_P)]),
    "sa_bsattn_fwd_plan": (_I, [_P, _P, _P, _P, _P, _P, _I, _F, _P]),
    "sa_bsattn_fwd_f32out": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P]),
    "sa_bsattn_fwd_noalloc": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P]),
    "sa_bsattn_fwd_plan_f32out": (_I, [_P, _P, _P, _P, _P, _P, _I, _F, _P]),
    "sa_bsattn_plan_stats": (_I, [_P, ctypes.POINTER(ctypes.c_int64)]),
    "sa_bsattn_plan_destroy": (_I, [_P]),
    "sa_dense_attn_fwd": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _P]),
    "sa_mask_instantiate": (_I, [_P, _P, _I, _I, _I, _I, _P, _P]),
    "sa_bsattn_fwd_layout": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _I, _P]),
    "sa_resize_mask": (_I, [_P, _I, _I, _I, _P, _I, _I, _P]),
    "sa_resize_threshold_map": (_I, [_P, _I, _I, _I, _P, _I, _I, _P]),
    "sa_fidelity_profile": (_I, [_P, _P, _P, _I, _P, _P, _I, _P, _P, _P, _I, _I, _I, _I, _I, _F,
                                 _P]),
    "sa_qk_norm_rope": (_I, [_P, _S, _P, _S, _P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I,
                             _F, _I, _I, _P]),
    "sa_qk_norm_rope_bwd_workspace": (_Z, [_I]),
    "sa_qk_norm_rope_bwd": (_I, [_P, _P, _P, _S, _P, _S, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I,
                                 _I, _I, _I, _I, _I, _I, _F, _I, _I, _P]),
    "sa_block_means": (_I, [_P, _S, _P, _I, _I, _I, _I, _I, _P]),
    "sa_block_select": (_I, [_P, _P, _P, _I, _P, _I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _P]),
    "sa_selected_attn_workspace": (_Z, [_I, _I, _I, _I, _I, _I]),
    "sa_selected_attn_fwd": (_I, [_P, _P, _P, _P, _I, _P, _I, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I,
                                  _I, _F, _P]),
    "sa_bsattn_bwd_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "sa_bsattn_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F,
                           _I, _P]),
    "sa_selected_decode_workspace": (_Z, [_I, _I, _I, _I, _I, _I, _I]),
    "sa_selected_decode": (_I, [_P, _P, _P, _S, _P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _I,
                                _F, _P]),
}


class SAError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (fn, status_string(status), status))


def library_path():
    return _build.LIB_PATH


def load(build_if_missing=True):
    """Load the library (building it in-tree only if it is absent)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        if not build_if_missing:
            raise RuntimeError("HIP library %s is not built" % path)
        _build.build()
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def status_string(status):
    return load().sa_status_string(int(status)).decode()


def _check(fn, status):
    if status != SA_OK:
        raise SAError(fn, status)


# --------------------------------------------------------------- tensors ---

def _torch():
    import torch
    return torch


def _dev_ptr(t, dtype, name):
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)
    if t.device.type != "cuda":
        raise ValueError("%s must be on the GPU, got %s" % (name, t.device))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return ctypes.c_void_p(t.data_ptr())


def _need(cond, msg):
    """Size checks on the host: the C ABI takes raw pointers and cannot see buffer sizes."""
    if not cond:
        raise ValueError(msg)


def _same_shape(ref, others, names):
    for t, n in zip(others, names):
        _need(tuple(t.shape) == tuple(ref.shape), "%s has shape %s, expected %s"
              % (n, tuple(t.shape), tuple(ref.shape)))


def _outputs(q, out, lse, lse_shape, out_dtype=None):
    torch = _torch()
    if out is None:
        out = torch.empty_like(q, dtype=out_dtype or q.dtype)
    _need(tuple(out.shape) == tuple(q.shape), "out must have the shape of q")
    if lse is None:
        lse = torch.empty(lse_shape, dtype=torch.float32, device=q.device)
    _need(tuple(lse.shape) == tuple(lse_shape), "lse must have shape %s" % (tuple(lse_shape),))
    return out, lse


def _mask_words(m, H, n_qb, n_kb):
    _need(m.numel() == H * n_qb * ((n_kb + 63) // 64),
          "mask has %d words, expected H * n_qb * ceil(n_kb / 64) = %d"
          % (m.numel(), H * n_qb * ((n_kb + 63) // 64)))


def _stream(stream):
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _used_on(stream, *tensors):
    """Tensors made here and used by work on a stream other than the current one:
    the caching allocator must not hand their memory out again before that
    stream's work on them is done (it only tracks the current stream by itself)."""
    if stream is None:
        return
    torch = _torch()
    if stream == torch.cuda.current_stream():
        return
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def mask_to_device(mask_bits, device="cuda"):
    """uint64 numpy [H, n_qb, W] -> int64 torch tensor (same bits) on ``device``."""
    torch = _torch()
    if isinstance(mask_bits, torch.Tensor):
        return mask_bits.to(device).contiguous()
    m = np.ascontiguousarray(mask_bits, dtype=np.uint64).view(np.int64)
    return torch.from_numpy(m.copy()).to(device)


def _fwd_oneshot(fn, out_dtype, q, k, v, mask_bits, blk_q, blk_k, scale, out, lse, stream):
    torch = _torch()
    lib = load()
    B, H, N, d = q.shape
    _same_shape(q, (k, v), ("k", "v"))
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    m = mask_to_device(mask_bits, q.device)
    if m.dtype == torch.uint64:
        m = m.view(torch.int64)
    _mask_words(m, H, -(-N // int(blk_q)), -(-N // int(blk_k)))
    out, lse = _outputs(q, out, lse, (B, H, N), out_dtype)
    st = getattr(lib, fn)(
        _dev_ptr(q, torch.bfloat16, "q"), _dev_ptr(k, torch.bfloat16, "k"),
        _dev_ptr(v, torch.bfloat16, "v"), _dev_ptr(m, torch.int64, "mask_bits"),
        _dev_ptr(out, out_dtype, "out"), _dev_ptr(lse, torch.float32, "lse"),
        B, H, N, d, int(blk_q), int(blk_k), float(scale), _stream(stream))
    _check(fn, st)
    _used_on(stream, m, out, lse)
    return out, lse


def bsattn_fwd(q, k, v, mask_bits, blk_q, blk_k, scale=None, out=None, lse=None, stream=None):
    """One-shot forward: ``sa_bsattn_fwd``.  q, k, v: bf16 [B, H, N, d] on the GPU.

    mask_bits: int64/uint64 device tensor (or numpy uint64) [H, n_qb, W].
    Returns (out bf16 [B, H, N, d], lse float32 [B, H, N]).
    """
    return _fwd_oneshot("sa_bsattn_fwd", _torch().bfloat16, q, k, v, mask_bits, blk_q, blk_k,
                        scale, out, lse, stream)


def bsattn_fwd_f32out(q, k, v, mask_bits, blk_q, blk_k, scale=None, out=None, lse=None,
                      stream=None):
    """``sa_bsattn_fwd_f32out``: as ``bsattn_fwd`` with out float32 [B, H, N, d]."""
    return _fwd_oneshot("sa_bsattn_fwd_f32out", _torch().float32, q, k, v, mask_bits, blk_q,
                        blk_k, scale, out, lse, stream)


def bsattn_fwd_bnhd(q, k, v, mask_bits, blk_q, blk_k, scale=None, out=None, lse=None,
                    stream=None):
    """``sa_bsattn_fwd_layout`` with q, k, v, out in [B, N, H, d]; lse is [B, H, N]."""
    torch = _torch()
    lib = load()
    B, N, H, d = q.shape
    _same_shape(q, (k, v), ("k", "v"))
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    m = mask_to_device(mask_bits, q.device)
    if m.dtype == torch.uint64:
        m = m.view(torch.int64)
    _mask_words(m, H, -(-N // int(blk_q)), -(-N // int(blk_k)))
    out, lse = _outputs(q, out, lse, (B, H, N))
    st = lib.sa_bsattn_fwd_layout(
        _dev_ptr(q, torch.bfloat16, "q"), _dev_ptr(k, torch.bfloat16, "k"),
        _dev_ptr(v, torch.bfloat16, "v"), _dev_ptr(m, torch.int64, "mask_bits"),
        _dev_ptr(out, torch.bfloat16, "out"), _dev_ptr(lse, torch.float32, "lse"),
        B, H, N, d, int(blk_q), int(blk_k), float(scale), SA_LAYOUT_BNHD, _stream(stream))
    _check("sa_bsattn_fwd_layout", st)
    _used_on(stream, m, out, lse)
    return out, lse


def dense_attn_fwd(q, k, v, blk=128, scale=None, out=None, lse=None, stream=None):
    """``sa_dense_attn_fwd``: maskless attention (every key block enabled).

    Up to 512 query blocks over batches and heads the bits of ``bsattn_fwd`` with an all-ones
    mask; beyond, its result to within rounding (the header gives the line)."""
    torch = _torch()
    lib = load()
    B, H, N, d = q.shape
    _same_shape(q, (k, v), ("k", "v"))
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    out, lse = _outputs(q, out, lse, (B, H, N))
    st = lib.sa_dense_attn_fwd(
        _dev_ptr(q, torch.bfloat16, "q"), _dev_ptr(k, torch.bfloat16, "k"),
        _dev_ptr(v, torch.bfloat16, "v"), _dev_ptr(out, torch.bfloat16, "out"),
        _dev_ptr(lse, torch.float32, "lse"), B, H, N, d, int(blk), float(scale), _stream(stream))
    _check("sa_dense_attn_fwd", st)
    _used_on(stream, out, lse)
    return out, lse


def mask_instantiate(T, p, out=None, stream=None):
    """``sa_mask_instantiate``: CRM masks 1[T <= p] for every threshold set.

    T: float32 device tensor [H, n_qb, n_kb]; p: float32 device tensor [n_p, H].
    Returns int64 (uint64 bits) [n_p, H, n_qb, W].
    """
    torch = _torch()
    lib = load()
    H, n_qb, n_kb = T.shape
    n_p = p.shape[0]
    if tuple(p.shape) != (n_p, H):
        raise ValueError("p must be [n_p, H]")
    W = (n_kb + 63) // 64
    if out is None:
        out = torch.empty((n_p, H, n_qb, W), dtype=torch.int64, device=T.device)
    _need(out.numel() == n_p * H * n_qb * W, "out must hold n_p * H * n_qb * W words")
    st = lib.sa_mask_instantiate(_dev_ptr(T, torch.float32, "T"), _dev_ptr(p, torch.float32, "p"),
                                 n_p, H, n_qb, n_kb, _dev_ptr(out, torch.int64, "mask_bits"),
                                 _stream(stream))
    _check("sa_mask_instantiate", st)
    _used_on(stream, out)
    return out


def fidelity_profile(q, k, rows, T, p, blk, scale=None, stream=None):
    """``sa_fidelity_profile``: returns (hellinger [B,H,R,K], fidelity [B,H,K], blk_lse [B,H,R,n_kb]).

    rows: int32 device tensor [H, R]; T: float32 device [H, n_qb, n_kb]; p: float32 device [K].
    """
    torch = _torch()
    lib = load()
    B, H, N, d = q.shape
    _same_shape(q, (k,), ("k",))
    _need(rows.dim() == 2 and rows.shape[0] == H, "rows must be [H, R]")
    R = rows.shape[1]
    _need(p.dim() == 1, "p must be [K]")
    K = p.shape[0]
    n_kb = (N + blk - 1) // blk
    _need(tuple(T.shape) == (H, n_kb, n_kb), "T must be [H, n_qb, n_kb] = %s" % ((H, n_kb, n_kb),))
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    dev = q.device
    blk_lse = torch.empty((B, H, R, n_kb), dtype=torch.float32, device=dev)
    hel = torch.empty((B, H, R, K), dtype=torch.float32, device=dev)
    fid = torch.empty((B, H, K), dtype=torch.float32, device=dev)
    st = lib.sa_fidelity_profile(
        _dev_ptr(q, torch.bfloat16, "q"), _dev_ptr(k, torch.bfloat16, "k"),
        _dev_ptr(rows, torch.int32, "rows"), R, _dev_ptr(T, torch.float32, "T"),
        _dev_ptr(p, torch.float32, "p"), K, _dev_ptr(blk_lse, torch.float32, "blk_lse"),
        _dev_ptr(hel, torch.float32, "hellinger"), _dev_ptr(fid, torch.float32, "fidelity"),
        B, H, N, d, int(blk), float(scale), _stream(stream))
    _check("sa_fidelity_profile", st)
    _used_on(stream, blk_lse, hel, fid)
    return hel, fid, blk_lse


def resize_threshold_map(T, n_qb_out, n_kb_out, stream=None):
    """``sa_resize_threshold_map``: float32 [H, n_qb, n_kb] -> [H, n_qb_out, n_kb_out]."""
    torch = _torch()
    lib = load()
    H, n_qb, n_kb = T.shape
    out = torch.empty((H, n_qb_out, n_kb_out), dtype=torch.float32, device=T.device)
    st = lib.sa_resize_threshold_map(_dev_ptr(T, torch.float32, "T"), H, n_qb, n_kb,
                                     _dev_ptr(out, torch.float32, "T_out"), n_qb_out, n_kb_out,
                                     _stream(stream))
    _check("sa_resize_threshold_map", st)
    _used_on(stream, out)
    return out


def resize_mask(mask_bits, n_kb, n_qb_out, n_kb_out, stream=None):
    """``sa_resize_mask``: CRM int64 [H, n_qb, W] (n_kb key blocks) -> [H, n_qb_out, W_out]."""
    torch = _torch()
    lib = load()
    m = mask_to_device(mask_bits)
    if m.dtype == torch.uint64:
        m = m.view(torch.int64)
    H, n_qb, _ = m.shape
    _mask_words(m, H, n_qb, n_kb)
    out = torch.empty((H, n_qb_out, (n_kb_out + 63) // 64), dtype=torch.int64, device=m.device)
    st = lib.sa_resize_mask(_dev_ptr(m, torch.int64, "mask_bits"), H, n_qb, n_kb,
                            _dev_ptr(out, torch.int64, "mask_out"), n_qb_out, n_kb_out,
                            _stream(stream))
    _check("sa_resize_mask", st)
    _used_on(stream, m, out)
    return out


def mask_prepass(mask_bits, H, n_qb, n_kb, stream=None):
    """``sa_mask_prepass``: returns (counts int32 [H*n_qb], lists int32 [H*n_qb, n_kb])."""
    torch = _torch()
    lib = load()
    m = mask_to_device(mask_bits, mask_bits.device if isinstance(mask_bits, torch.Tensor) else "cuda")
    if m.dtype == torch.uint64:
        m = m.view(torch.int64)
    _mask_words(m, H, n_qb, n_kb)
    counts = torch.full((H * n_qb,), -1, dtype=torch.int32, device=m.device)
    lists = torch.full((H * n_qb, n_kb), -1, dtype=torch.int32, device=m.device)
    st = lib.sa_mask_prepass(_dev_ptr(m, torch.int64, "mask_bits"), H, n_qb, n_kb,
                             _dev_ptr(counts, torch.int32, "counts"),
                             _dev_ptr(lists, torch.int32, "lists"), _stream(stream))
    _check("sa_mask_prepass", st)
    _used_on(stream, m, counts, lists)
    return counts, lists


def schedule(counts, B, H, n_qb, stream=None):
    """``sa_schedule``: returns order int32 [B*H*n_qb]."""
    torch = _torch()
    lib = load()
    _need(counts.numel() == H * n_qb, "counts must hold H * n_qb entries")
    order = torch.full((B * H * n_qb,), -1, dtype=torch.int32, device=counts.device)
    st = lib.sa_schedule(_dev_ptr(counts, torch.int32, "counts"), B, H, n_qb,
                         _dev_ptr(order, torch.int32, "order"), _stream(stream))
    _check("sa_schedule", st)
    _used_on(stream, order)
    return order


def bsattn_fwd_prepared(q, k, v, counts, lists, order, blk_q, blk_k, scale=None, out=None,
                        lse=None, stream=None):
    """``sa_bsattn_fwd_prepared``: attention kernel on a given pre-pass and schedule."""
    torch = _torch()
    lib = load()
    B, H, N, d = q.shape
    _same_shape(q, (k, v), ("k", "v"))
    n_qb, n_kb = -(-N // int(blk_q)), -(-N // int(blk_k))
    _need(counts.numel() == H * n_qb, "counts must hold H * n_qb entries")
    _need(lists.numel() == H * n_qb * n_kb, "lists must hold H * n_qb * n_kb entries")
    _need(order.numel() == B * H * n_qb, "order must hold B * H * n_qb entries")
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    out, lse = _outputs(q, out, lse, (B, H, N))
    st = lib.sa_bsattn_fwd_prepared(
        _dev_ptr(q, torch.bfloat16, "q"), _dev_ptr(k, torch.bfloat16, "k"),
        _dev_ptr(v, torch.bfloat16, "v"), _dev_ptr(counts, torch.int32, "counts"),
        _dev_ptr(lists, torch.int32, "lists"), _dev_ptr(order, torch.int32, "order"),
        _dev_ptr(out, torch.bfloat16, "out"), _dev_ptr(lse, torch.float32, "lse"),
        B, H, N, d, int(blk_q), int(blk_k), float(scale), _stream(stream))
    _check("sa_bsattn_fwd_prepared", st)
    _used_on(stream, out, lse)
    return out, lse


class Plan:
    """Static-mask plan (``sa_bsattn_plan_*``): pre-pass and schedule done once."""

    def __init__(self, mask_bits, B, H, N, blk_q, blk_k, stream=None):
        torch = _torch()
        self._lib = load()
        self._m = mask_to_device(mask_bits)
        if self._m.dtype == torch.uint64:
            self._m = self._m.view(torch.int64)
        _mask_words(self._m, H, -(-N // int(blk_q)), -(-N // int(blk_k)))
        self.B, self.H, self.N, self.blk_q, self.blk_k = B, H, N, blk_q, blk_k
        h = ctypes.c_void_p()
        st = self._lib.sa_bsattn_plan_create(_dev_ptr(self._m, torch.int64, "mask_bits"), B, H, N,
                                             blk_q, blk_k, _stream(stream), ctypes.byref(h))
        _check("sa_bsattn_plan_create", st)
        self._h = h

    @property
    def executed_blocks(self):
        n = ctypes.c_int64()
        _check("sa_bsattn_plan_stats", self._lib.sa_bsattn_plan_stats(self._h, ctypes.byref(n)))
        return n.value

    def _fwd(self, fn, out_dtype, q, k, v, scale, out, lse, stream):
        torch = _torch()
        B, H, N, d = q.shape
        if (B, H, N) != (self.B, self.H, self.N):
            raise ValueError("q shape %s does not match the plan" % (tuple(q.shape),))
        _same_shape(q, (k, v), ("k", "v"))
        if scale is None:
            scale = 1.0 / float(d) ** 0.5
        out, lse = _outputs(q, out, lse, (B, H, N), out_dtype)
        st = getattr(self._lib, fn)(
            self._h, _dev_ptr(q, torch.bfloat16, "q"), _dev_ptr(k, torch.bfloat16, "k"),
            _dev_ptr(v, torch.bfloat16, "v"), _dev_ptr(out, out_dtype, "out"),
            _dev_ptr(lse, torch.float32, "lse"), d, float(scale), _stream(stream))
        _check(fn, st)
        _used_on(stream, out, lse)
        return out, lse

    def __call__(self, q, k, v, scale=None, out=None, lse=None, stream=None):
        """``sa_bsattn_fwd_plan``: (out bf16 [B, H, N, d], lse float32 [B, H, N])."""
        return self._fwd("sa_bsattn_fwd_plan", _torch().bfloat16, q, k, v, scale, out, lse,
                         stream)

    def fwd_f32out(self, q, k, v, scale=None, out=None, lse=None, stream=None):
        """``sa_bsattn_fwd_plan_f32out``: as the call, with out float32."""
        return self._fwd("sa_bsattn_fwd_plan_f32out", _torch().float32, q, k, v, scale, out, lse,
                         stream)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.sa_bsattn_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------- around the attention ---
#
# Tensors may be on any GPU, all on the same one; the work goes to that GPU's
# current stream, or to ``stream``, which has to be of that GPU and then waits
# for the current one (the functions above leave that wait to the caller).  Inputs
# that the caller frees before ``stream`` is done with them need
# ``Tensor.record_stream`` there, as with the functions above.  The checks are
# written for small calls, which take the host longer than the GPU.

_PAIRS = {"interleaved": SA_PAIRS_INTERLEAVED, "halves": SA_PAIRS_HALVES}
_LAYOUTS = {"bhnd": SA_LAYOUT_BHND, "bnhd": SA_LAYOUT_BNHD}


def _named(table, key, name):
    if key not in table:
        raise ValueError("%s must be one of %s, got %r" % (name, ", ".join(sorted(table)), key))
    return table[key]


def _device(t, name):
    """Index of the GPU that the call's first tensor is on."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU, got %s" % (name, t.device))
    return t.get_device()


def _ptr(t, dtype, name, dev):
    """Address of a contiguous tensor on GPU ``dev``."""
    if not (isinstance(t, _torch().Tensor) and t.dtype == dtype and t.is_contiguous()):
        _dev_ptr(t, dtype, name)  # raises
    if t.get_device() != dev and _device(t, name) != dev:
        raise ValueError("%s is on GPU %d, others are on GPU %d" % (name, t.get_device(), dev))
    return t.data_ptr()


def _ptrs(dev, dtype, **named):
    """Addresses of contiguous tensors of one type on GPU ``dev``; None stays None."""
    out = []
    for name, t in named.items():
        if t is None:
            out.append(None)
            continue
        try:
            good = t.dtype is dtype and t.is_contiguous() and t.get_device() == dev
        except AttributeError:
            good = False
        out.append(t.data_ptr() if good else _ptr(t, dtype, name, dev))
    return out


@functools.lru_cache(maxsize=256)
def _strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def _rows_ptr(t, name, dev):
    """Address and strides of bf16 rows whose last dimension is contiguous; the strides of the
    others (any order, 0 for a repeated row) in the tensor's order."""
    if _device(t, name) != dev:
        raise ValueError("%s is on GPU %d, others are on GPU %d" % (name, t.get_device(), dev))
    if t.dtype is not _torch().bfloat16:
        raise TypeError("%s must be %s, got %s" % (name, _torch().bfloat16, t.dtype))
    if t.dim() != 4:
        raise ValueError("%s must have four dimensions, got %d" % (name, t.dim()))
    (n0, n1, n2, n3), (s0, s1, s2, s3) = t.shape, t.stride()
    if max(n0, n1, n2) >= 1 << 31:  # the library's sizes are 32-bit numbers
        raise ValueError("%s has a dimension of %d" % (name, max(n0, n1, n2)))
    if s3 != 1 and n3 != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    # the stride of a dimension of one entry means nothing
    s0, s1, s2 = s0 if n0 > 1 else 0, s1 if n1 > 1 else 0, s2 if n2 > 1 else 0
    ptr = t.data_ptr()
    if (s0 | s1 | s2) % 8 or ptr % 16:
        raise ValueError("%s: rows must be 16-byte aligned" % name)
    return ptr, _strides(s0, s1, s2)


def _run(fn, dev, stream, args, made):
    """Calls ``fn`` with GPU ``dev`` current, on its current stream or ``stream``; ``made`` are the
    tensors allocated for the call."""
    torch = _torch()
    if stream is None and torch.cuda.current_device() == dev:
        st = getattr(_LIB or load(), fn)(*args, _current_stream(dev))
    else:
        _need(stream is None or stream.device_index == dev, "stream is of another GPU")
        with torch.cuda.device(dev):
            now = torch.cuda.current_stream()
            if stream is not None and stream != now:
                stream.wait_stream(now)  # the inputs, and who had the new tensors' memory before
            st = getattr(load(), fn)(*args, (stream or now).cuda_stream)
            _used_on(stream, *made)
    if st != SA_OK:
        raise SAError(fn, st)


def _topk(topk):
    topk = int(topk)
    if not 1 <= topk < 1 << 31:
        raise ValueError("topk must be at least 1 and a 32-bit number, got %d" % topk)
    return topk


def _current_stream(dev):
    """Handle of the current stream of GPU ``dev``; torch's own launchers ask for it this way, a
    Stream object takes 2.6 us to make."""
    torch = _torch()
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(dev) if get else torch.cuda.current_stream(dev).cuda_stream


def _workspace(like, fn, *sizes):
    """A workspace for the call, None where it needs none (or refuses the sizes)."""
    n = getattr(_LIB or load(), fn)(*sizes)
    return like.new_empty(n, dtype=_torch().uint8) if n else None


def _address(t):
    return None if t is None else t.data_ptr()


def _mask_arg(m, B, H, n_qb, n_kb, name):
    """int64 bits [H, n_qb, W] or [1 or B, H, n_qb, W]; returns (tensor, its batches)."""
    torch = _torch()
    if m is None:
        return None, 1
    if not isinstance(m, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)
    if m.dtype == torch.uint64:
        m = m.view(torch.int64)
    shape = (H, n_qb, (n_kb + 63) // 64)
    if m.shape == shape:
        return m, 1
    if m.shape != (1,) + shape and m.shape != (B,) + shape:
        raise ValueError("%s has shape %s, expected %s, alone or for each batch entry"
                         % (name, tuple(m.shape), shape))
    return m, m.shape[0]


def _rope_shapes(q, k, wq, wk, cos, sin, positions, pairs, layout):
    _need(q.dim() == 4 and k.dim() == 4, "q and k must be [B, N, heads, d]")
    B, N, Hq, d = q.shape
    B2, N2, Hk, d2 = k.shape
    if not (B2 == B and N2 == N and d2 == d):
        raise ValueError("k has shape %s, expected [%d, %d, heads, %d]" % (tuple(k.shape), B, N, d))
    _need(wq.shape == (d,) and wk.shape == (d,), "wq and wk must be [d]")
    _need(cos.dim() == 2 and cos.shape == sin.shape, "cos and sin must be [positions, rot / 2]")
    n_pos, half = cos.shape
    if n_pos >= 1 << 31:
        raise ValueError("cos and sin have %d positions" % n_pos)
    if positions is not None:
        _need(positions.shape == (B, N), "positions must be [B, N]")
    elif n_pos < N:
        raise ValueError("cos and sin have %d positions for %d tokens" % (n_pos, N))
    return (B, N, Hq, Hk, d, 2 * half, n_pos, _named(_PAIRS, pairs, "pairs"),
            _named(_LAYOUTS, layout, "layout"))


def _heads_shape(layout, B, N, H, d):
    return (B, H, N, d) if layout == SA_LAYOUT_BHND else (B, N, H, d)


def qk_norm_rope(q, k, wq, wk, cos, sin, positions=None, eps=1e-6, pairs="interleaved",
                 layout="bhnd", stream=None):
    """``sa_qk_norm_rope``: every head's RMS norm and the rotation by position.

    q, k: bf16 [B, N, Hq or Hk, d], the first three dimensions of any strides (slices of one
    projection's output); wq, wk: float32 [d]; cos, sin: float32 [positions, rot / 2];
    positions: int32 [B, N], None for 0 .. N - 1.  Returns q and k in bf16, [B, H, N, d]
    (``layout`` "bhnd", as the attention reads them) or [B, N, H, d] ("bnhd").
    """
    torch = _torch()
    dev = _device(q, "q")
    q_ptr, q_str = _rows_ptr(q, "q", dev)
    k_ptr, k_str = _rows_ptr(k, "k", dev)
    ptrs = _ptrs(dev, torch.float32, wq=wq, wk=wk, cos=cos, sin=sin)
    pos = None if positions is None else _ptr(positions, torch.int32, "positions", dev)
    B, N, Hq, Hk, d, rot, n_pos, pr, lay = _rope_shapes(q, k, wq, wk, cos, sin, positions, pairs,
                                                        layout)
    q_out = q.new_empty(_heads_shape(lay, B, N, Hq, d))
    k_out = q.new_empty(_heads_shape(lay, B, N, Hk, d))
    _run("sa_qk_norm_rope", dev, stream,
         (q_ptr, q_str, k_ptr, k_str, *ptrs, pos, q_out.data_ptr(), k_out.data_ptr(), B, N, Hq, Hk, d, rot,
          n_pos, eps, pr, lay), (q_out, k_out))
    return q_out, k_out


def qk_norm_rope_bwd(dq_out, dk_out, q, k, wq, wk, cos, sin, positions=None, eps=1e-6,
                     pairs="interleaved", layout="bhnd", stream=None):
    """``sa_qk_norm_rope_bwd``: gradients of ``qk_norm_rope`` with respect to q, k, wq and wk.

    dq_out, dk_out: bf16, contiguous, in the layout of the forward's outputs.  Returns
    (dq bf16 [B, N, Hq, d], dk bf16 [B, N, Hk, d], dwq float32 [d], dwk float32 [d]).
    """
    torch = _torch()
    dev = _device(q, "q")
    q_ptr, q_str = _rows_ptr(q, "q", dev)
    k_ptr, k_str = _rows_ptr(k, "k", dev)
    grads = _ptrs(dev, torch.bfloat16, dq_out=dq_out, dk_out=dk_out)
    ptrs = _ptrs(dev, torch.float32, wq=wq, wk=wk, cos=cos, sin=sin)
    pos = None if positions is None else _ptr(positions, torch.int32, "positions", dev)
    B, N, Hq, Hk, d, rot, n_pos, pr, lay = _rope_shapes(q, k, wq, wk, cos, sin, positions, pairs,
                                                        layout)
    for t, H, name in ((dq_out, Hq, "dq_out"), (dk_out, Hk, "dk_out")):
        if t.shape != _heads_shape(lay, B, N, H, d):
            raise ValueError("%s has shape %s, expected %s"
                             % (name, tuple(t.shape), _heads_shape(lay, B, N, H, d)))
    dq, dk = q.new_empty((B, N, Hq, d)), q.new_empty((B, N, Hk, d))
    dwq, dwk = wq.new_empty(d), wq.new_empty(d)
    ws = _workspace(q, "sa_qk_norm_rope_bwd_workspace", d)
    _run("sa_qk_norm_rope_bwd", dev, stream,
         (*grads, q_ptr, q_str, k_ptr, k_str, *ptrs, pos, dq.data_ptr(), dk.data_ptr(), dwq.data_ptr(),
          dwk.data_ptr(), _address(ws), B, N, Hq, Hk, d, rot, n_pos, eps, pr, lay),
         (dq, dk, dwq, dwk, ws))
    return dq, dk, dwq, dwk


def block_means(x, blk, stream=None):
    """``sa_block_means``: float32 [B, H, ceil(N / blk), d], the means of blocks of blk tokens.

    x: bf16 [B, H, N, d], the first three dimensions of any strides (a transposed
    [B, N, H, d], or the tokens of a cache's newly finished block).
    """
    dev = _device(x, "x")
    _need(x.dim() == 4, "x must be [B, H, N, d]")
    ptr, strides = _rows_ptr(x, "x", dev)
    B, H, N, d = x.shape
    _need(blk in (64, 128), "blk must be 64 or 128")
    means = x.new_empty((B, H, -(-N // blk), d), dtype=_torch().float32)
    _run("sa_block_means", dev, stream, (ptr, strides, means.data_ptr(), B, H, N, d, blk), (means,))
    return means


def block_select(q_means, k_means, topk, candidates=None, keep=None, stream=None):
    """``sa_block_select``: mask bits int64 [B, H, n_qb, W] of the topk best key blocks of every
    query block by the products of their means (float32 [B, H, n_qb, d] and [B, H, n_kb, d]).

    candidates: mask bits that choices are limited to; keep: blocks that every row has beside
    them.  Each int64 [H, n_qb, W], shared by the batch, or [B, H, n_qb, W].
    """
    torch = _torch()
    dev = _device(q_means, "q_means")
    ptrs = _ptrs(dev, torch.float32, q_means=q_means, k_means=k_means)
    _need(q_means.dim() == 4 and k_means.dim() == 4, "q_means and k_means must be [B, H, blocks, d]")
    B, H, n_qb, d = q_means.shape
    B2, H2, n_kb, d2 = k_means.shape
    if not (B2 == B and H2 == H and d2 == d):
        raise ValueError("k_means has shape %s, expected [%d, %d, blocks, %d]"
                         % (tuple(k_means.shape), B, H, d))
    candidates, cb = _mask_arg(candidates, B, H, n_qb, n_kb, "candidates")
    keep, kb = _mask_arg(keep, B, H, n_qb, n_kb, "keep")
    c_ptr, k_ptr = _ptrs(dev, torch.int64, candidates=candidates, keep=keep)
    mask = q_means.new_empty((B, H, n_qb, (n_kb + 63) // 64), dtype=torch.int64)
    _run("sa_block_select", dev, stream,
         (*ptrs, c_ptr, cb, k_ptr, kb, mask.data_ptr(), None, None, B, H, n_qb, n_kb, d, _topk(topk)),
         (mask,))
    return mask


def selected_attn_fwd(q, k, v, blk_q, blk_k, topk, candidates=None, keep=None, scale=None,
                      stream=None):
    """``sa_selected_attn_fwd``: block means of q and k, the selection of ``block_select``, and the
    attention over it.  q, k, v: bf16 [B, H, N, d].

    Returns (out bf16 [B, H, N, d], lse float32 [B, H, N], mask bits int64 [B, H, n_qb, W]);
    the mask is what ``bsattn_bwd`` takes.
    """
    torch = _torch()
    dev = _device(q, "q")
    ptrs = _ptrs(dev, torch.bfloat16, q=q, k=k, v=v)
    _need(q.dim() == 4, "q must be [B, H, N, d]")
    B, H, N, d = q.shape
    if not (k.shape == v.shape == q.shape):
        _same_shape(q, (k, v), ("k", "v"))
    _need(blk_q in (64, 128) and blk_k in (64, 128), "blk_q and blk_k must be 64 or 128")
    n_qb, n_kb = -(-N // blk_q), -(-N // blk_k)
    candidates, cb = _mask_arg(candidates, B, H, n_qb, n_kb, "candidates")
    keep, kb = _mask_arg(keep, B, H, n_qb, n_kb, "keep")
    c_ptr, k_ptr = _ptrs(dev, torch.int64, candidates=candidates, keep=keep)
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    out = q.new_empty((B, H, N, d))
    lse = q.new_empty((B, H, N), dtype=torch.float32)
    mask = q.new_empty((B, H, n_qb, (n_kb + 63) // 64), dtype=torch.int64)
    ws = _workspace(q, "sa_selected_attn_workspace", B, H, N, d, blk_q, blk_k)
    _run("sa_selected_attn_fwd", dev, stream,
         (*ptrs, c_ptr, cb, k_ptr, kb, out.data_ptr(), lse.data_ptr(), mask.data_ptr(), _address(ws),
          B, H, N, d, blk_q, blk_k, _topk(topk), scale),
         (out, lse, mask, ws))
    return out, lse, mask


def bsattn_bwd(dout, q, k, v, out, lse, mask_bits, blk_q, blk_k, scale=None, layout="bhnd",
               stream=None):
    """``sa_bsattn_bwd``: (dq, dk, dv) of the attention through a block mask held fixed.

    dout, q, k, v, out: bf16 [B, H, N, d], or [B, N, H, d] with ``layout`` "bnhd"; out and lse
    (float32 [B, H, N]) of the forward pass with the same arguments.  mask_bits: int64 bits
    [H, n_qb, W] as ``bsattn_fwd`` takes them (numpy too), or [B, H, n_qb, W] as
    ``selected_attn_fwd`` returns them.
    """
    torch = _torch()
    dev = _device(q, "q")
    ptrs = _ptrs(dev, torch.bfloat16, dout=dout, q=q, k=k, v=v, out=out)
    ptrs += _ptrs(dev, torch.float32, lse=lse)
    lay = _named(_LAYOUTS, layout, "layout")
    _need(q.dim() == 4, "q must have four dimensions")
    if lay == SA_LAYOUT_BHND:
        B, H, N, d = q.shape
    else:
        B, N, H, d = q.shape
    if not (dout.shape == k.shape == v.shape == out.shape == q.shape):
        _same_shape(q, (dout, k, v, out), ("dout", "k", "v", "out"))
    _need(lse.shape == (B, H, N), "lse must be [B, H, N]")
    _need(blk_q in (64, 128) and blk_k in (64, 128), "blk_q and blk_k must be 64 or 128")
    if not isinstance(mask_bits, torch.Tensor):
        mask_bits = mask_to_device(mask_bits, q.device)
    m, batches = _mask_arg(mask_bits, B, H, -(-N // blk_q), -(-N // blk_k), "mask_bits")
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    dq, dk, dv = q.new_empty(q.shape), q.new_empty(q.shape), q.new_empty(q.shape)
    ws = _workspace(q, "sa_bsattn_bwd_workspace", B, H, N, d, blk_q, blk_k, batches)
    _run("sa_bsattn_bwd", dev, stream,
         (*ptrs, _ptr(m, torch.int64, "mask_bits", dev), batches, dq.data_ptr(), dk.data_ptr(),
          dv.data_ptr(), _address(ws), B, H, N, d, blk_q, blk_k, scale, lay), (m, dq, dk, dv, ws))
    return dq, dk, dv


def selected_decode(q, k, v, means, lengths, topk, blk, scale=None, stream=None):
    """``sa_selected_decode``: attention of one token a sequence over the topk blocks of its cache
    that the means of their keys select, the newest token's among them.

    q: bf16 [B, Hq, d]; k, v: bf16 [B, Hkv, cap, d], the first three dimensions of any strides,
    both alike, the newest token already in them; means: float32 [B, Hkv, ceil(cap / blk), d],
    right for the blocks before the newest token's; lengths: int32 [B], tokens in the cache.
    Returns (out bf16 [B, Hq, d], lse float32 [B, Hq], blocks int32 [B, Hkv, topk]).
    """
    torch = _torch()
    dev = _device(q, "q")
    q_ptr = _ptr(q, torch.bfloat16, "q", dev)
    _need(q.dim() == 3 and k.dim() == 4, "q must be [B, Hq, d], k and v [B, Hkv, cap, d]")
    k_ptr, strides = _rows_ptr(k, "k", dev)
    v_ptr, v_strides = _rows_ptr(v, "v", dev)
    B, Hq, d = q.shape
    B2, Hkv, cap, d2 = k.shape
    topk = _topk(topk)
    if not (B2 == B and d2 == d and Hkv > 0 and Hq % Hkv == 0):
        raise ValueError("k has shape %s, q %s" % (tuple(k.shape), tuple(q.shape)))
    if v.shape != k.shape:
        raise ValueError("v has shape %s, expected %s" % (tuple(v.shape), tuple(k.shape)))
    _need(strides is v_strides or strides[:] == v_strides[:], "k and v must have the same strides")
    _need(blk in (64, 128), "blk must be 64 or 128")
    if means.shape != (B, Hkv, -(-cap // blk), d):
        raise ValueError("means must have shape %s" % ((B, Hkv, -(-cap // blk), d),))
    _need(lengths.shape == (B,), "lengths must be [B]")
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    out = q.new_empty((B, Hq, d))
    lse = q.new_empty((B, Hq), dtype=torch.float32)
    blocks = q.new_empty((B, Hkv, topk), dtype=torch.int32)
    ws = _workspace(q, "sa_selected_decode_workspace", B, Hq, Hkv, cap, d, blk, topk)
    _run("sa_selected_decode", dev, stream,
         (q_ptr, k_ptr, v_ptr, strides, _ptr(means, torch.float32, "means", dev),
          _ptr(lengths, torch.int32, "lengths", dev), out.data_ptr(), lse.data_ptr(), blocks.data_ptr(),
          _address(ws), B, Hq, Hkv, cap, d, blk, topk, scale), (out, lse, blocks, ws))
    return out, lse, blocks
