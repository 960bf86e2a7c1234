"""Sizes whose launches HIP does not take (2^32 threads or more) are refused on the host by the
operators around the attention, before anything is enqueued; the sizes just below are not."""

import pytest

from paper_2606_23019_amd import binding
from test_operator_refusals import FakeGpu, bwd, decode, means, select, selected, strides

UNSUPPORTED = binding.SA_ERR_UNSUPPORTED
M = 1 << 20


@pytest.mark.parametrize("d,line", [(128, 2 * M), (64, 4 * M)])
def test_gradients_of_more_rows_than_a_launch_takes(lib, d, line):
    # 1024 threads for every 64 (d = 128) or 128 (d = 64) padded tokens
    for B, H in ((line, 1), (1, line), (line // 8, 8), (2 * line, 1)):
        assert lib.sa_bsattn_bwd_workspace(B, H, 1, d, 64, 64, 1) == 0
        assert bwd(lib, B=B, H=H, N=1, d=d) == UNSUPPORTED
    assert lib.sa_bsattn_bwd_workspace(line - 64, 1, 1, d, 64, 64, 1) > 0


@pytest.mark.parametrize("blk", [64, 128])
def test_means_of_more_blocks_than_a_launch_takes(lib, blk):
    for kw in (dict(B=16 * M, H=1, N=1), dict(B=1, H=M, N=16 * blk), dict(B=4, H=1, N=4 * M * blk - 7)):
        assert means(lib, s=strides(64, 64, 64), blk=blk, **kw) == UNSUPPORTED


def test_selections_of_more_rows_than_a_launch_takes(lib):
    # 512 threads for 16 rows; for one row where a row's keys fill LDS
    assert select(lib, B=1, H=1, n_qb=128 * M, n_kb=7) == UNSUPPORTED
    assert select(lib, B=1, H=1, n_qb=8 * M, n_kb=16384) == UNSUPPORTED
    assert select(lib, B=8 * M, H=1, n_qb=1, n_kb=1) == UNSUPPORTED


def test_attention_over_a_selection_of_more_rows_than_a_launch_takes(lib):
    for B, H in ((8 * M, 1), (1, 8 * M)):
        assert lib.sa_selected_attn_workspace(B, H, 1, 64, 64, 64) == 0
        assert selected(lib, B=B, H=H, N=1) == UNSUPPORTED
    assert lib.sa_selected_attn_workspace(8 * M - 64, 1, 1, 64, 64, 64) > 0


def test_workspace_of_a_refused_selection_is_zero(lib):
    assert lib.sa_selected_attn_workspace(1, 1, 64 * 16384, 64, 64, 64) > 0
    assert lib.sa_selected_attn_workspace(1, 1, 64 * 16385, 64, 64, 64) == 0


def test_norm_and_rotation_of_more_rows_than_a_launch_takes(lib):
    # 256 threads for 16 tokens of up to 16 heads; addresses 2^40 apart, past the tensors' ends
    def call(N):
        a = [binding.ctypes.c_void_p(i << 40) for i in range(1, 9)]
        s = strides(0, 128, 128)
        return lib.sa_qk_norm_rope(a[0], s, a[1], s, a[2], a[3], a[4], a[5], None, a[6], a[7], 1, N, 1, 1,
                                   128, 128, N, 1e-6, 0, 0, None)
    assert call(128 * M) == UNSUPPORTED


def test_decode_of_more_scores_than_a_launch_takes(lib):
    # 512 threads for 256 blocks of a row's table, where tables are long
    assert lib.sa_selected_decode_workspace(M // 8, 1, 1, 16384 * 64, 64, 64, 99) == 0
    assert decode(lib, B=M // 8, Hq=1, Hkv=1, cap=16384 * 64, d=64, topk=99, s=strides(0, 0, 0)) == UNSUPPORTED
    assert lib.sa_selected_decode_workspace(M // 8 - 1, 1, 1, 16384 * 64, 64, 64, 99) > 0


def test_binding_refuses_sizes_beyond_32_bits():
    """The C ABI's sizes are ints: a larger one would arrive as another number."""
    import torch
    row = FakeGpu(torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16))
    n = (1 << 32) + 64
    for shape in ((n, 1, 1, 64), (1, n, 1, 64), (1, 1, n, 64), (1, 1, 1 << 31, 64)):
        with pytest.raises(ValueError, match="x has a dimension of"):
            binding._rows_ptr(row.expand(shape), "x", 0)
    assert list(binding._rows_ptr(row.expand(1, 1, (1 << 31) - 1, 64), "x", 0)[1]) == [0, 0, 0]
    w = torch.zeros(64)
    cos = torch.zeros((1, 32)).expand((1 << 32) + 1, 32)
    with pytest.raises(ValueError, match="cos and sin have"):
        binding._rope_shapes(row, row, w, w, cos, cos, torch.zeros((1, 1)).int(), "halves", "bhnd")


def test_norm_and_rotation_of_more_heads_than_a_kernel_counts(lib):
    # a run of heads ends up to 16 past H, in an int
    def call(Hq, Hk, bwd):
        a = [binding.ctypes.c_void_p(i << 44) for i in range(1, 15)]
        s = strides(0, 0, 0)
        tail = (1, 1, Hq, Hk, 64, 64, 1, 1e-6, 0, 0, None)
        if bwd:
            return lib.sa_qk_norm_rope_bwd(a[0], a[1], a[2], s, a[3], s, a[4], a[5], a[6], a[7], None, a[8], a[9],
                                           a[10], a[11], a[12], *tail)
        return lib.sa_qk_norm_rope(a[0], s, a[1], s, a[2], a[3], a[4], a[5], None, a[6], a[7], *tail)
    for bwd in (False, True):
        for heads in ((1 << 30) + 1, (1 << 31) - 2):
            assert call(heads, 1, bwd) == UNSUPPORTED and call(1, heads, bwd) == UNSUPPORTED
