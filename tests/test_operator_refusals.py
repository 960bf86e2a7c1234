"""Bad arguments of the operators around the attention are refused on the host (no GPU here): the
C ABI by its status before any HIP call, the binding by what it raises."""

import ctypes

import pytest

from paper_2606_23019_amd import binding

P = ctypes.c_void_p
INVALID, UNSUPPORTED = binding.SA_ERR_INVALID_ARG, binding.SA_ERR_UNSUPPORTED
A, MB = 1 << 40, 1 << 30  # fake device addresses, far apart: every call below is refused


def at(i):
    return A + i * MB


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def rope(lib, bwd=False, q=at(0), k=at(1), wq=at(2), cos=at(3), sin=at(4), positions=0,
         q_out=at(5), k_out=at(6), B=2, N=100, Hq=4, Hk=2, d=128, rot=128, n_pos=100, eps=1e-6,
         pairs=0, layout=0, qs=None, dw=at(9), ws=at(10)):
    qs = qs or strides(N * Hq * d, Hq * d, d)
    ks = strides(N * Hk * d, Hk * d, d)
    tail = (B, N, Hq, Hk, d, rot, n_pos, eps, pairs, layout, None)
    if bwd:
        return lib.sa_qk_norm_rope_bwd(P(q_out), P(k_out), P(q), qs, P(k), ks, P(wq), P(at(11)), P(cos),
                                       P(sin), P(positions), P(at(7)), P(at(8)), P(dw), P(at(12)),
                                       P(ws), *tail)
    return lib.sa_qk_norm_rope(P(q), qs, P(k), ks, P(wq), P(at(11)), P(cos), P(sin), P(positions),
                               P(q_out), P(k_out), *tail)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(q=0), INVALID), (dict(wq=0), INVALID), (dict(cos=0), INVALID), (dict(k_out=0), INVALID),
    (dict(q=at(0) + 8), INVALID), (dict(cos=at(3) + 8), INVALID), (dict(q_out=at(5) + 4), INVALID),
    (dict(B=0), INVALID), (dict(N=0), INVALID), (dict(Hk=0), INVALID), (dict(n_pos=99), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(pairs=2), INVALID),
    (dict(layout=2), INVALID), (dict(d=96), UNSUPPORTED), (dict(rot=130), UNSUPPORTED),
    (dict(rot=24), UNSUPPORTED), (dict(rot=0), UNSUPPORTED), (dict(rot=144), UNSUPPORTED),
    (dict(qs=strides(-8, 512, 128)), INVALID), (dict(qs=strides(51200, 516, 128)), INVALID),
    (dict(qs=strides(1 << 62, 512, 128)), INVALID),
    (dict(B=1 << 16, N=1 << 16, n_pos=1 << 16), UNSUPPORTED),
])
def test_rope_refuses(lib, bwd, kw, code):
    assert rope(lib, bwd, **kw) == code


def test_rope_refuses_overlaps(lib):
    assert rope(lib, q_out=at(0) + 64) == INVALID
    assert rope(lib, q_out=at(6) + 64) == INVALID
    assert rope(lib, q_out=at(0) + 2 * 99 * 4 * 128 * 2) == INVALID  # q's second batch entry
    assert rope(lib, True, ws=at(7)) == INVALID
    assert rope(lib, True, ws=0) == INVALID and rope(lib, True, dw=0) == INVALID
    assert lib.sa_qk_norm_rope_bwd_workspace(96) == 0


def means(lib, x=at(0), s=None, m=at(1), B=1, H=2, N=300, d=128, blk=128):
    return lib.sa_block_means(P(x), s or strides(H * N * d, N * d, d), P(m), B, H, N, d, blk, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), INVALID), (dict(m=0), INVALID), (dict(x=at(0) + 2), INVALID), (dict(N=0), INVALID),
    (dict(s=strides(0, 0, 4)), INVALID), (dict(d=32), UNSUPPORTED), (dict(blk=32), UNSUPPORTED),
    (dict(m=at(0) + 16), INVALID), (dict(N=(1 << 31) - 1, s=strides(0, 0, 0)), UNSUPPORTED),
])
def test_means_refuse(lib, kw, code):
    assert means(lib, **kw) == code


def select(lib, qm=at(0), km=at(1), cand=0, cb=1, keep=0, kb=1, bits=at(2), counts=0, lists=0, B=2, H=3,
           n_qb=5, n_kb=7, d=64, topk=2):
    return lib.sa_block_select(P(qm), P(km), P(cand), cb, P(keep), kb, P(bits), P(counts), P(lists), B,
                               H, n_qb, n_kb, d, topk, None)


@pytest.mark.parametrize("kw,code", [
    (dict(qm=0), INVALID), (dict(bits=0), INVALID), (dict(bits=at(2) + 4), INVALID),
    (dict(topk=0), INVALID), (dict(n_kb=0), INVALID), (dict(n_kb=16385), UNSUPPORTED),
    (dict(d=32), UNSUPPORTED), (dict(counts=at(3)), INVALID), (dict(cand=at(3), cb=3), INVALID),
    (dict(keep=at(3), kb=0), INVALID), (dict(cand=at(3) + 4), INVALID), (dict(bits=at(0)), INVALID),
    (dict(cand=at(2)), INVALID), (dict(H=1 << 30), UNSUPPORTED),
])
def test_select_refuses(lib, kw, code):
    assert select(lib, **kw) == code


def selected(lib, q=at(0), v=at(2), cand=0, cb=1, out=at(3), lse=at(4), bits=at(5), ws=at(6), B=2, H=3,
             N=300, d=64, bq=64, bk=64, topk=2, scale=0.1):
    return lib.sa_selected_attn_fwd(P(q), P(at(1)), P(v), P(cand), cb, None, 1, P(out), P(lse), P(bits),
                                    P(ws), B, H, N, d, bq, bk, topk, scale, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), INVALID), (dict(ws=0), INVALID), (dict(ws=at(6) + 16), INVALID), (dict(topk=0), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(d=80), UNSUPPORTED),
    (dict(bq=96), UNSUPPORTED), (dict(N=64 * 16385), UNSUPPORTED), (dict(out=at(0) + 16), INVALID),
    (dict(lse=at(6) + 64), INVALID), (dict(cand=at(7), cb=4), INVALID), (dict(B=0), INVALID),
])
def test_selected_refuses(lib, kw, code):
    assert selected(lib, **kw) == code


def bwd(lib, dout=at(0), q=at(1), out=at(4), lse=at(5), m=at(6), mb=1, dq=at(7), dv=at(9), ws=at(10),
        B=2, H=3, N=300, d=64, bq=64, bk=64, scale=0.1, layout=0):
    return lib.sa_bsattn_bwd(P(dout), P(q), P(at(2)), P(at(3)), P(out), P(lse), P(m), mb, P(dq),
                             P(at(8)), P(dv), P(ws), B, H, N, d, bq, bk, scale, layout, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dout=0), INVALID), (dict(m=0), INVALID), (dict(q=at(1) + 8), INVALID),
    (dict(lse=at(5) + 2), INVALID), (dict(ws=at(10) + 128), INVALID), (dict(mb=3), INVALID),
    (dict(mb=0), INVALID), (dict(layout=5), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=1e-31), INVALID), (dict(N=0), INVALID),
    (dict(d=256), UNSUPPORTED), (dict(bk=256), UNSUPPORTED), (dict(dq=at(0)), INVALID),
    (dict(dv=at(7) + 16), INVALID), (dict(ws=at(5)), INVALID),
    (dict(layout=1, H=1 << 16, d=128), UNSUPPORTED), (dict(N=64 * 65536), UNSUPPORTED),
])
def test_bwd_refuses(lib, kw, code):
    assert bwd(lib, **kw) == code


def decode(lib, q=at(0), k=at(1), s=None, means=at(3), lengths=at(4), out=at(5), blocks=at(7), ws=at(8),
           B=2, Hq=8, Hkv=2, cap=1000, d=128, blk=64, topk=4, scale=0.1):
    return lib.sa_selected_decode(P(q), P(k), P(at(2)), s or strides(Hkv * cap * d, cap * d, d), P(means),
                                  P(lengths), P(out), P(at(6)), P(blocks), P(ws), B, Hq, Hkv, cap, d, blk,
                                  topk, scale, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), INVALID), (dict(means=0), INVALID), (dict(lengths=0), INVALID), (dict(ws=0, topk=99), INVALID),
    (dict(k=at(1) + 8), INVALID), (dict(Hq=9), INVALID), (dict(topk=0), INVALID), (dict(cap=0), INVALID),
    (dict(d=96), UNSUPPORTED), (dict(blk=16), UNSUPPORTED), (dict(cap=64 * 16385), UNSUPPORTED),
    (dict(s=strides(0, 0, 129)), INVALID), (dict(out=at(0)), INVALID), (dict(blocks=at(5) + 64), INVALID),
    (dict(ws=at(1) + 256, topk=99), INVALID), (dict(scale=float("inf")), INVALID),
])
def test_decode_refuses(lib, kw, code):
    assert decode(lib, **kw) == code


def test_workspaces_of_refused_sizes_are_zero(lib):
    assert lib.sa_selected_attn_workspace(1, 1, 0, 64, 64, 64) == 0
    assert lib.sa_bsattn_bwd_workspace(2, 1, 64, 64, 64, 64, 3) == 0
    assert lib.sa_selected_decode_workspace(1, 3, 2, 64, 64, 64, 1) == 0
    assert lib.sa_selected_decode_workspace(1, 2, 2, 64, 64, 64, 1) == 0  # needs none
    assert lib.sa_selected_decode_workspace(1, 2, 2, 10000, 64, 64, 99) > 0
    assert lib.sa_bsattn_bwd_workspace(1, 1, 64, 64, 64, 64, 1) % 256 == 0


def FakeGpu(t, index=0):
    """A tensor that says it is on a GPU."""
    import torch

    class OnGpu(torch.Tensor):
        is_cuda = True
        device = torch.device("cuda", index)

        def get_device(self):
            return index
    return t.as_subclass(OnGpu)


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    x = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        binding.block_means(x, 64)
    with pytest.raises(TypeError):
        binding.block_means([1.0], 64)
    with pytest.raises(ValueError, match="on the GPU"):
        binding.bsattn_bwd(x, x, x, x, x, x, torch.zeros((2, 1, 1), dtype=torch.int64), 64, 64)
    with pytest.raises(ValueError, match="on the GPU"):
        binding._ptr(x, torch.bfloat16, "x", 0)
    with pytest.raises(TypeError, match="must be torch.float32"):
        binding._ptr(FakeGpu(x), torch.float32, "x", 0)
    with pytest.raises(ValueError, match="contiguous"):
        binding._ptr(FakeGpu(x.transpose(1, 2)), torch.bfloat16, "x", 0)
    with pytest.raises(ValueError, match="is on GPU 1"):
        binding._ptr(FakeGpu(x, 1), torch.bfloat16, "x", 0)
    with pytest.raises(ValueError, match="is on GPU 1"):
        binding._rows_ptr(FakeGpu(x, 1), "x", 0)
    assert binding._ptr(FakeGpu(x), torch.bfloat16, "x", 0) == x.data_ptr()
    with pytest.raises(ValueError, match="four dimensions"):
        binding._rows_ptr(FakeGpu(x[0]), "x", 0)
    for topk in (0, -1, 1 << 31, (1 << 32) + 1):
        with pytest.raises(ValueError, match="topk must be"):
            binding._topk(topk)
    with pytest.raises(ValueError, match="pairs must be"):
        binding._named(binding._PAIRS, "both", "pairs")
    for shape in ((1, 1, 1), (2, 2, 1), (2, 3, 1, 1), (2, 1, 1, 1, 1)):
        with pytest.raises(ValueError, match="mask_bits has shape"):
            binding._mask_arg(torch.zeros(shape, dtype=torch.int64), 3, 2, 1, 1, "mask_bits")
    for ok, n in (((2, 1, 1), 1), ((1, 2, 1, 1), 1), ((3, 2, 1, 1), 3)):
        assert binding._mask_arg(torch.zeros(ok, dtype=torch.int64), 3, 2, 1, 1, "mask_bits")[1] == n
    with pytest.raises(ValueError, match="16-byte"):
        binding._rows_ptr(FakeGpu(torch.zeros((1, 4, 2, 65), dtype=torch.bfloat16)[..., :64]), "x", 0)
    with pytest.raises(ValueError, match="last dimension"):
        binding._rows_ptr(FakeGpu(x.transpose(2, 3)), "x", 0)
    assert list(binding._rows_ptr(FakeGpu(x.transpose(1, 2)), "x", 0)[1]) == [0, 64, 128]
    assert list(binding._rows_ptr(FakeGpu(x[:, :1].expand(3, 4, 2, 64)), "x", 0)[1]) == [0, 0, 64]
