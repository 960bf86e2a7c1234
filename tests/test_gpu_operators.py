"""The operators around the attention on the GPU against their float64 reference.

Tolerances: a result in bf16 is off by its rounding, half a step (U16 of the value), and by what the
fp32 arithmetic before it adds, which oracle.operators bounds from the inputs; probabilities and score
gradients are rounded to bf16 for the products, U16 each."""

import numpy as np
import pytest

from oracle import operators as ops

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, scale=1.0):
    import torch
    return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()


def check(got, ref, bound):
    got = f64(got)
    assert got.shape == ref.shape
    err, allowed = np.abs(got - ref), bound + U16 * (np.abs(ref) + bound)
    bad = ~(err <= allowed)
    assert not bad.any(), "%d of %d, worst %.3g of %.3g allowed at %s" % (
        bad.sum(), bad.size, err[bad].max(), allowed[bad][0], np.argwhere(bad)[0])


def unpack(bits, n_kb):
    w = f64_bits(bits)
    return ((w[..., None] >> np.arange(64, dtype=np.uint64)) & np.uint64(1)).astype(bool).reshape(
        *w.shape[:-1], -1)[..., :n_kb]


def f64_bits(t):
    return t.cpu().numpy().view(np.uint64)


def pack(on):
    import torch
    n = on.shape[-1]
    full = np.zeros(on.shape[:-1] + (-(-n // 64) * 64,), dtype=bool)
    full[..., :n] = on
    words = (full.reshape(*on.shape[:-1], -1, 64).astype(np.uint64) << np.arange(64, dtype=np.uint64)).sum(
        -1, dtype=np.uint64)
    return torch.from_numpy(words.view(np.int64).copy()).cuda()


# ------------------------------------------------------ norm and rotation ---

ROPE = [  # B, N, Hq, Hk, d, rot, pairs, layout, positions, fused
    (1, 1, 1, 1, 128, 128, "interleaved", "bhnd", False, False),
    (1, 1, 1, 1, 64, 64, "halves", "bnhd", True, False),
    (3, 1, 40, 8, 128, 128, "halves", "bnhd", True, True),
    (2, 77, 6, 3, 64, 32, "halves", "bhnd", False, True),
    (2, 77, 6, 3, 64, 48, "halves", "bhnd", True, False),
    (1, 333, 5, 1, 128, 48, "interleaved", "bhnd", True, True),
    (1, 333, 5, 1, 128, 16, "halves", "bnhd", False, False),
    (2, 1000, 33, 17, 128, 128, "interleaved", "bhnd", False, True),
    (1, 4097, 20, 20, 64, 64, "interleaved", "bnhd", False, False),
]


def rope_inputs(case, seed):
    import torch
    B, N, Hq, Hk, d, rot, pairs, layout, positions, fused = case
    g = gen(seed)
    if fused:
        x = randn(g, B, N, Hq + 2 * Hk, d)
        q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hk]
    else:
        q, k = randn(g, B, N, Hq, d), randn(g, B, N, Hk, d, scale=3.0)
    q[:, ::5] = 0  # rows of zeros: eps alone keeps them finite
    wq, wk = (1 + 0.3 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
    n_pos = 2 * N + 3 if positions else N
    angle = torch.rand((n_pos, rot // 2), generator=g, device="cuda", dtype=torch.float64) * 6.3
    cos, sin = angle.cos().float(), angle.sin().float()
    pos = torch.randint(n_pos, (B, N), generator=g, device="cuda").int() if positions else None
    at = (pos.cpu().numpy() if positions else np.broadcast_to(np.arange(N), (B, N)))
    return q, k, wq, wk, cos, sin, pos, f64(cos)[at], f64(sin)[at]


@pytest.mark.parametrize("case", ROPE)
def test_norm_rope(case):
    from paper_2606_23019_amd import binding
    B, N, Hq, Hk, d, rot, pairs, layout, positions, fused = case
    q, k, wq, wk, cos, sin, pos, c, s = rope_inputs(case, 11)
    eps = 1e-5
    got = binding.qk_norm_rope(q, k, wq, wk, cos, sin, positions=pos, eps=eps, pairs=pairs, layout=layout)
    for y, x, w in zip(got, (q, k), (wq, wk)):
        assert y.is_contiguous()
        y = y.transpose(1, 2) if layout == "bhnd" else y
        # both products of a turned element are at most sqrt(d) max w; d + 16 roundings each
        bound = 2 * (d + 16) * U32 * d ** 0.5 * float(w.abs().max())
        check(y, ops.norm_rope(f64(x), f64(w), c, s, eps, pairs), bound)


@pytest.mark.parametrize("case", ROPE)
def test_norm_rope_bwd(case):
    from paper_2606_23019_amd import binding
    B, N, Hq, Hk, d, rot, pairs, layout, positions, fused = case
    q, k, wq, wk, cos, sin, pos, c, s = rope_inputs(case, 12)
    g, eps = gen(13), 1e-2
    grads = [randn(g, *((B, H, N, d) if layout == "bhnd" else (B, N, H, d))) for H in (Hq, Hk)]
    got = binding.qk_norm_rope_bwd(*grads, q, k, wq, wk, cos, sin, positions=pos, eps=eps, pairs=pairs,
                                   layout=layout)
    again = binding.qk_norm_rope_bwd(*grads, q, k, wq, wk, cos, sin, positions=pos, eps=eps, pairs=pairs,
                                     layout=layout)
    for dx, dw, dy, x, w, dx2, dw2 in zip(got[:2], got[2:], grads, (q, k), (wq, wk), again[:2], again[2:]):
        assert (dx == dx2).all() and (dw == dw2).all()
        dy = f64(dy.transpose(1, 2) if layout == "bhnd" else dy)
        x, w = f64(x), f64(w)
        rx, rw = ops.norm_rope_grad(dy, x, w, c, s, eps, pairs)
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        # g w of a turned pair, and n mean(w g n) with mean of |w g n| at most its rms: d + 16 roundings
        size = np.abs(dy).max(-1, keepdims=True) * 1.5 * np.abs(w).max()
        n = np.abs(x) * r
        check(dx, rx, 2 * (d + 16) * U32 * r * size * (1 + n * n.mean(-1, keepdims=True)))
        # dw: d + 16 roundings of each term, and one for each of the sum's (at most 2^12 a lane)
        terms = (1.5 * np.abs(dy).max(-1, keepdims=True) * n).sum((0, 1, 2))
        err = np.abs(f64(dw) - rw)
        assert (err <= (d + 16 + min(4096, B * N * max(Hq, Hk))) * U32 * terms).all(), err.max()


def test_norm_rope_strides_and_positions_out_of_range():
    import torch
    from paper_2606_23019_amd import binding
    g = gen(5)
    x = randn(g, 2, 3, 9, 7, 128)  # heads before tokens, and a batch of which one entry is repeated
    q, k = x[0].transpose(1, 2), x[1, :1].transpose(1, 2).expand(3, 7, 9, 128)
    w = torch.ones(128, device="cuda")
    cos, sin = (torch.rand((5, 64), generator=g, device="cuda") for _ in range(2))
    pos = torch.tensor([[-3, 0, 1, 2, 3, 4, 99]] * 3, device="cuda", dtype=torch.int32)
    got = binding.qk_norm_rope(q, k, w, w, cos, sin, positions=pos)
    ref = binding.qk_norm_rope(q.contiguous(), k.contiguous(), w, w, cos, sin, positions=pos.clamp(0, 4))
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_norm_rope_past_the_caches():
    """More than the last cache holds is read and written past it: the same results."""
    import torch
    from paper_2606_23019_amd import binding
    B, N, H, d = 2, 12000, 26, 128
    q, k, wq, wk, cos, sin, _, _, _ = rope_inputs((B, N, H, H, d, d, "halves", "bhnd", False, True), 3)
    assert 2 * B * N * H * d * 2 > 256 << 20
    got = binding.qk_norm_rope(q, k, wq, wk, cos, sin, pairs="halves")
    dq, dk, _, _ = binding.qk_norm_rope_bwd(*got, q, k, wq, wk, cos, sin, pairs="halves")
    for b in range(B):
        part = q[b:b + 1], k[b:b + 1], wq, wk, cos, sin
        ref = binding.qk_norm_rope(*part, pairs="halves")
        assert all(torch.equal(x[b:b + 1], y) for x, y in zip(got, ref))
        ref = binding.qk_norm_rope_bwd(got[0][b:b + 1], got[1][b:b + 1], *part, pairs="halves")
        assert torch.equal(dq[b:b + 1], ref[0]) and torch.equal(dk[b:b + 1], ref[1])
    x = torch.cat([q, k], 2).transpose(1, 2).repeat(1, 2, 1, 1)
    means = binding.block_means(x, 64)
    assert torch.equal(means[:, :H], binding.block_means(q.transpose(1, 2), 64))
    assert torch.equal(means[:, -H:], binding.block_means(k.transpose(1, 2), 64))


# --------------------------------------------------------------- selection ---

@pytest.mark.parametrize("B,H,N,d,blk", [(1, 1, 1, 128, 128), (2, 3, 200, 64, 64), (1, 2, 1000, 128, 64),
                                         (1, 1, 129, 64, 128), (2, 1, 640, 128, 128)])
def test_block_means(B, H, N, d, blk):
    import torch
    from paper_2606_23019_amd import binding
    x = randn(gen(N), B, N, H, d) * 100
    x[:, ::3] = 1e-4
    got = binding.block_means(x.transpose(1, 2), blk)
    ref = ops.block_means(f64(x.transpose(1, 2)), blk)
    # summed in 64 bits and rounded once
    assert (np.abs(f64(got) - ref) <= U32 * np.abs(ref) + 1e-12).all()
    assert torch.equal(got, binding.block_means(x.transpose(1, 2).contiguous(), blk))


SELECT = [  # B, H, n_qb, n_kb, d, topk, candidates, keep
    (1, 1, 1, 1, 64, 1, None, None), (1, 2, 17, 63, 128, 5, None, "shared"),
    (2, 2, 16, 64, 64, 64, "own", None), (1, 3, 5, 65, 128, 70, "shared", "own"),
    (1, 1, 33, 300, 64, 1, None, None), (2, 1, 20, 641, 128, 60, "own", "shared"),
    (1, 1, 19, 1290, 64, 100, None, None), (1, 1, 3, 9001, 64, 33, "shared", None),
    (1, 1, 2, 16384, 128, 700, None, None),
]


@pytest.mark.parametrize("case", SELECT)
def test_block_select(case):
    import torch
    from paper_2606_23019_amd import binding
    B, H, n_qb, n_kb, d, topk, cand, keep = case
    g = gen(n_kb)
    qm, km = (torch.randn((B, H, n, d), generator=g, device="cuda") for n in (n_qb, n_kb))
    km[:, :, n_kb // 2:] = km[:, :, :n_kb - n_kb // 2].clone()  # every score twice
    rng = np.random.default_rng(n_kb)

    def bits(kind, p):
        if kind is None:
            return None, [[None] * H] * B
        on = rng.random((B if kind == "own" else 1, H, n_qb, n_kb)) < p
        on[:, 0, 0] = False  # a row with no candidate, or nothing kept
        return pack(on if kind == "own" else on[0]), [[on[b % len(on), h] for h in range(H)]
                                                      for b in range(B)]
    cb, con = bits(cand, 0.5)
    kb, kon = bits(keep, 0.03)
    got = unpack(binding.block_select(qm, km, topk, candidates=cb, keep=kb), n_kb)
    for b in range(B):
        for h in range(H):
            ref = ops.block_select(f64(qm[b, h]), f64(km[b, h]), topk, con[b][h], kon[b][h])
            assert np.array_equal(got[b, h], ref), (b, h, np.argwhere(got[b, h] != ref)[:4])


def test_block_select_of_special_values():
    import torch
    from paper_2606_23019_amd import binding
    inf, nan = float("inf"), float("nan")
    km = torch.zeros((1, 1, 70, 64), device="cuda")
    km[0, 0, :, 0] = torch.tensor([nan, -inf, 0.0, -0.0, inf, 1e-40, nan] + [-1.0] * 63)
    qm = torch.zeros((1, 1, 1, 64), device="cuda")
    qm[..., 0] = 1.0
    order = [4, 5, 2, 3] + list(range(7, 70)) + [1, 0, 6]
    for topk in (1, 2, 3, 4, 5, 66, 67, 68, 69, 70, 71):
        on = unpack(binding.block_select(qm, km, topk), 70)[0, 0, 0]
        assert sorted(order[:topk]) == list(np.nonzero(on)[0]), topk


def test_block_select_lists_are_the_mask_s():
    import torch
    import ctypes
    from paper_2606_23019_amd import binding
    lib, P = binding.load(), ctypes.c_void_p
    B, H, n_qb, n_kb, d = 2, 2, 7, 150, 64
    g = gen(1)
    qm, km = (torch.randn((B, H, n, d), generator=g, device="cuda") for n in (n_qb, n_kb))
    mask = torch.empty((B, H, n_qb, 3), dtype=torch.int64, device="cuda")
    counts = torch.full((B * H * n_qb,), -1, dtype=torch.int32, device="cuda")
    lists = torch.full((B * H * n_qb, n_kb), -1, dtype=torch.int32, device="cuda")
    assert lib.sa_block_select(P(qm.data_ptr()), P(km.data_ptr()), None, 1, None, 1, P(mask.data_ptr()),
                               P(counts.data_ptr()), P(lists.data_ptr()), B, H, n_qb, n_kb, d, 9,
                               binding._stream(None)) == 0
    rc, rl = binding.mask_prepass(mask.view(B * H, n_qb, 3), B * H, n_qb, n_kb)
    assert torch.equal(counts, rc) and torch.equal(lists, rl)


@pytest.mark.parametrize("B,H,N,d,blk_q,blk_k,topk", [
    (1, 1, 1, 64, 64, 64, 1), (2, 3, 700, 128, 64, 64, 4), (2, 2, 1100, 64, 128, 64, 5),
    (1, 4, 900, 128, 128, 128, 3), (2, 9, 2000, 64, 64, 128, 6), (1, 20, 2100, 128, 128, 128, 5)])
def test_selected_attn(B, H, N, d, blk_q, blk_k, topk):
    import torch
    from paper_2606_23019_amd import binding
    g = gen(N)
    q, k, v = (randn(g, B, H, N, d) for _ in range(3))
    n_qb, n_kb = -(-N // blk_q), -(-N // blk_k)
    rng = np.random.default_rng(N)
    cand = rng.random((H, n_qb, n_kb)) < 0.7
    cand[:, n_qb // 2] = False  # rows with nothing
    out, lse, mask = binding.selected_attn_fwd(q, k, v, blk_q, blk_k, topk, candidates=pack(cand))
    ref = binding.block_select(binding.block_means(q, blk_q), binding.block_means(k, blk_k), topk,
                               candidates=pack(cand))
    assert torch.equal(mask, ref)
    heads = [t.view(1, B * H, N, d) for t in (q, k, v)]
    o2, l2 = binding.bsattn_fwd(*heads, mask.view(B * H, n_qb, -1), blk_q, blk_k)
    assert torch.equal(out.view(-1), o2.view(-1)) and torch.equal(lse.view(-1), l2.view(-1))
    assert torch.isneginf(lse[:, :, n_qb // 2 * blk_q]).all() and (out[:, :, n_qb // 2 * blk_q] == 0).all()


# --------------------------------------------------------------- gradients ---

BWD = [  # B, H, N, d, blk_q, blk_k, density, layout, a mask for every batch entry, input scale
    (1, 1, 1, 128, 128, 128, 1.0, "bhnd", False, 1.0),
    (1, 1, 1, 64, 64, 64, 1.0, "bnhd", False, 1.0),
    (1, 2, 64, 128, 64, 64, 1.0, "bhnd", False, 1.0),
    (1, 2, 65, 64, 128, 64, 1.0, "bhnd", False, 1.0),
    (2, 2, 200, 128, 128, 128, 0.6, "bhnd", True, 1.5),
    (2, 3, 333, 64, 64, 128, 0.5, "bnhd", True, 1.0),
    (1, 2, 449, 128, 64, 128, 0.4, "bnhd", False, 2.0),
    (2, 2, 600, 128, 128, 64, 0.4, "bhnd", False, 1.0),
    (1, 3, 800, 64, 64, 64, 0.3, "bnhd", False, 2.0),
    (1, 9, 1025, 128, 128, 128, 0.3, "bhnd", False, 1.0),
    (2, 2, 1216, 64, 128, 128, 0.2, "bnhd", True, 1.0),
]


@pytest.mark.parametrize("case", BWD)
def test_bsattn_bwd(case):
    import torch
    from paper_2606_23019_amd import binding
    B, H, N, d, blk_q, blk_k, rho, layout, own, size = case
    g = gen(N + d)
    shape = (B, H, N, d) if layout == "bhnd" else (B, N, H, d)
    q, k, v = (randn(g, *shape, scale=size) for _ in range(3))
    dout = randn(g, *shape)
    n_qb, n_kb = -(-N // blk_q), -(-N // blk_k)
    rng = np.random.default_rng(N)
    on = rng.random((B if own else 1, H, n_qb, n_kb)) < rho
    if n_qb > 2:
        on[:, :, 1] = False  # query blocks that see nothing
        on[:, :, :, n_kb - 1] = False  # a key block that nothing sees
        on[:, -1, :, 0] = True
        on[:, -1, n_qb - 1, n_kb - 1] = True  # the ragged corner
    if H > 2:
        on[:, 1] = False  # a head without any pair
    heads = (lambda t: t) if layout == "bhnd" else (lambda t: t.transpose(1, 2))
    out, lse = torch.empty_like(q), torch.empty((B, H, N), device="cuda")
    for b in range(B):  # the forward call has one mask for all of its batch entries
        fwd = binding.bsattn_fwd if layout == "bhnd" else binding.bsattn_fwd_bnhd
        o, l = fwd(*(t[b:b + 1].contiguous() for t in (q, k, v)), pack(on[b if own else 0]), blk_q, blk_k)
        out[b], lse[b] = o[0], l[0]
    mask = pack(on if own else on[0])
    got = binding.bsattn_bwd(dout, q, k, v, out, lse, mask, blk_q, blk_k, layout=layout)
    again = binding.bsattn_bwd(dout, q, k, v, out, lse, mask, blk_q, blk_k, layout=layout)
    for a, b2 in zip(got, again):
        assert a.is_contiguous() and torch.equal(a, b2)
    scale = d ** -0.5
    for b in range(B):
        for h in range(H):
            see = on[b if own else 0, h].repeat(blk_q, 0)[:N].repeat(blk_k, 1)[:, :N]
            x = [f64(heads(t)[b, h]) for t in (dout, q, k, v, out)]
            ref, bound = ops.attention_grad(*x, f64(lse[b, h]), see, scale, U16)
            for t, r, e in zip(got, ref, bound):
                check(heads(t)[b, h], r, e)
            assert not ref[0][~see.any(1)].any() and not f64(heads(got[0])[b, h])[~see.any(1)].any()
            assert not f64(heads(got[1])[b, h])[~see.any(0)].any()
            assert not f64(heads(got[2])[b, h])[~see.any(0)].any()


def test_bsattn_bwd_of_many_heads():
    """More items than the plan holds at once: the heads' results are those of smaller calls, bit
    for bit (no list is long enough to be cut in either)."""
    import torch
    from paper_2606_23019_amd import binding
    H, N, d, blk = 576, 3840, 64, 64
    n = N // blk
    g = gen(9)
    q, k, v, dout = (randn(g, 1, H, N, d) for _ in range(4))
    on = np.random.default_rng(9).random((H, n, n)) < 0.08
    mask = pack(on)
    out, lse = binding.bsattn_fwd(q, k, v, mask, blk, blk)
    got = binding.bsattn_bwd(dout, q, k, v, out, lse, mask, blk, blk)
    for h0 in (0, 300):
        h = slice(h0, h0 + 276)
        part = [t[:, h].contiguous() for t in (dout, q, k, v, out)]
        ref = binding.bsattn_bwd(*part, lse[:, h].contiguous(), mask[h].contiguous(), blk, blk)
        assert all(torch.equal(a[:, h], b) for a, b in zip(got, ref))


# ------------------------------------------------------------ single tokens ---

DECODE = [  # B, Hq, Hkv, cap, d, blk, topk, lengths
    (1, 1, 1, 1, 128, 64, 1, [1]),
    (3, 4, 4, 64, 64, 64, 2, [0, 1, 64]),
    (4, 8, 2, 300, 128, 128, 2, [300, 129, 128, 127]),
    (3, 16, 1, 1000, 128, 64, 5, [1000, 961, 960]),
    (2, 40, 2, 777, 64, 64, 1, [777, 65]),
    (2, 12, 3, 5000, 128, 64, 100, [5000, 4000]),
    (1, 32, 1, 3000, 64, 128, 7, [2999]),
    (2, 5, 1, 20000, 128, 64, 33, [20000, 15001]),
    (1, 1, 1, 100000, 64, 64, 20, [99999]),
    (2, 2, 1, 140001, 64, 64, 40, [140001, 70000]),
    (1, 2, 1, 320001, 64, 64, 40, [320001]),
]


@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("case", DECODE)
def test_selected_decode(case, tokens_first):
    import torch
    from paper_2606_23019_amd import binding
    B, Hq, Hkv, cap, d, blk, topk, lengths = case
    g = gen(cap)
    q = randn(g, B, Hq, d)
    shape = (B, cap, Hkv, d) if tokens_first else (B, Hkv, cap, d)
    k, v = randn(g, *shape), randn(g, *shape)
    if tokens_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    means = binding.block_means(k, blk)
    for b, n in enumerate(lengths):  # nothing past the last token is read
        k[b, :, n:], v[b, :, n:] = float("nan"), float("nan")
        means[b, :, max(0, -(-n // blk) - 1):] = float("nan")
    ln = torch.tensor(lengths, device="cuda", dtype=torch.int32)
    out, lse, blocks = binding.selected_decode(q, k, v, means, ln, topk, blk)
    again = binding.selected_decode(q, k, v, means, ln, topk, blk)
    assert all(torch.equal(a, b) for a, b in zip((out, lse, blocks), again))
    G = Hq // Hkv
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            rows = slice(h * G, (h + 1) * G)
            ro, rl, rb, eo, el = ops.selected_decode(f64(q[b, rows]), f64(k[b, h]), f64(v[b, h]),
                                                     f64(means[b, h]), n, topk, blk, d ** -0.5, U16)
            assert blocks[b, h].tolist() == rb + [-1] * (topk - len(rb))
            if n == 0:
                assert (out[b, rows] == 0).all() and torch.isneginf(lse[b, rows]).all()
                continue
            check(out[b, rows], ro, eo)
            assert (np.abs(f64(lse[b, rows]) - rl) <= el).all()


@pytest.mark.parametrize("B,cap,blk,topk", [(9, 8300, 128, 65), (70, 1024, 64, 16)])
def test_selected_decode_past_the_caches(B, cap, blk, topk):
    """Chosen blocks of more than the last cache holds, in parts and in one launch."""
    import torch
    from paper_2606_23019_amd import binding
    Hkv, G, d = 8, 2, 128
    assert B * Hkv * topk * blk * d * 4 > 256 << 20
    g = gen(cap)
    q, k, v = randn(g, B, Hkv * G, d), randn(g, B, Hkv, cap, d), randn(g, B, Hkv, cap, d)
    means = binding.block_means(k, blk)
    ln = torch.full((B,), cap - 3, device="cuda", dtype=torch.int32)
    out, lse, blocks = binding.selected_decode(q, k, v, means, ln, topk, blk)
    for b, h in ((0, 0), (B // 2, 3), (B - 1, Hkv - 1)):
        rows = slice(h * G, (h + 1) * G)
        ro, rl, rb, eo, el = ops.selected_decode(f64(q[b, rows]), f64(k[b, h]), f64(v[b, h]),
                                                 f64(means[b, h]), cap - 3, topk, blk, d ** -0.5, U16)
        assert blocks[b, h].tolist() == rb + [-1] * (topk - len(rb))
        check(out[b, rows], ro, eo)
        assert (np.abs(f64(lse[b, rows]) - rl) <= el).all()


def test_decode_lengths_out_of_range_are_clamped():
    import torch
    from paper_2606_23019_amd import binding
    g = gen(2)
    q, k, v = randn(g, 2, 2, 64), randn(g, 2, 1, 200, 64), randn(g, 2, 1, 200, 64)
    means = binding.block_means(k, 64)
    a = binding.selected_decode(q, k, v, means, torch.tensor([1000, -5], device="cuda").int(), 2, 64)
    b = binding.selected_decode(q, k, v, means, torch.tensor([200, 0], device="cuda").int(), 2, 64)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---------------------------------------------------------------- together ---

def chain(binding, x, w, tables, blk, topk):
    """A layer's attention from its projection's output, and the gradients back to it."""
    H = x.shape[2] // 3
    q, k = binding.qk_norm_rope(x[:, :, :H], x[:, :, H:2 * H], *w, *tables)
    v = x[:, :, 2 * H:].transpose(1, 2).contiguous()
    out, lse, mask = binding.selected_attn_fwd(q, k, v, blk, blk, topk)
    dq, dk, dv = binding.bsattn_bwd(out, q, k, v, out, lse, mask, blk, blk)
    return (out, lse, mask, dv) + binding.qk_norm_rope_bwd(dq, dk, x[:, :, :H], x[:, :, H:2 * H], *w,
                                                           *tables)


def chain_inputs(seed, B=2, N=900, H=3, d=128):
    import torch
    g = gen(seed)
    w = [1 + 0.1 * torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    angle = torch.rand((N, d // 2), generator=g, device="cuda") * 6.3
    return randn(g, B, N, 3 * H, d), w, (angle.cos(), angle.sin())


@pytest.mark.parametrize("N,blk", [(900, 128), (2500, 64)])
def test_chain_eager_other_stream_and_captured(N, blk):
    import torch
    from paper_2606_23019_amd import binding
    x, w, tables = chain_inputs(21, N=N)
    ref = chain(binding, x, w, tables, blk, 3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain(binding, x, w, tables, blk, 3)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    static = x.clone()
    graphs = []
    for _ in range(2):  # two graphs, each with its own memory, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, chain(binding, static, w, tables, blk, 3)))
        graphs[-1] = (graph, graphs[-1][1])
    for rep in range(3):
        new = chain_inputs(30 + rep, N=N)[0]
        want = chain(binding, new, w, tables, blk, 3)
        static.copy_(new)
        for graph, outs in graphs:
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            junk = (new.float() * 2).sum()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)) and torch.isfinite(junk)


def test_long_selections_and_decode_captured():
    """Selections whose keys take more LDS than a kernel has by itself, and every form of the
    single-token call, replayed in a graph on new inputs."""
    import torch
    from paper_2606_23019_amd import binding
    g = gen(50)

    def inputs():
        return [torch.randn((1, 2, n, 128), generator=g, device="cuda") for n in (33, 900)] + [
            randn(g, 2, 4, 64), randn(g, 2, 2, 140000, 64)]

    def calls(qm, km, q, k):
        outs = [binding.block_select(qm, km, 77)]
        for cap, topk in ((3000, 9), (60000, 70), (140000, 70)):  # one launch, chosen apart, scored apart
            kc = k[:, :, :cap]
            ln = torch.full((2,), cap - 5, device="cuda", dtype=torch.int32)
            outs += binding.selected_decode(q, kc, kc, binding.block_means(kc, 64), ln, topk, 64)
        return outs
    static = inputs()
    calls(*static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = calls(*static)
    for _ in range(3):
        new = inputs()
        want = calls(*new)
        for a, b in zip(static, new):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        junk = (new[0] * 2).sum()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)) and torch.isfinite(junk)


def test_stream_argument():
    """A call on another stream waits for what made its inputs on the current one."""
    import torch
    from paper_2606_23019_amd import binding
    x, w, tables = chain_inputs(22)
    ref = binding.qk_norm_rope(x[:, :, :3], x[:, :, 3:6], *w, *tables)
    side = torch.cuda.Stream()
    big = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        y = torch.zeros_like(x)
        for _ in range(8):
            big = (big @ big).clamp_(-1, 1)  # keeps the current stream busy before y is there
        y.copy_(x)
        got = binding.qk_norm_rope(y[:, :, :3], y[:, :, 3:6], *w, *tables, stream=side)
        y.record_stream(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_decode_continues_what_the_prompt_began():
    """Prompt by norm, rotation and selection, then tokens one by one into the cache: the first
    token's result is the prompt attention's over the same blocks."""
    import torch
    from paper_2606_23019_amd import binding
    B, H, d, blk, cap, N = 1, 2, 128, 64, 640, 500
    g = gen(40)
    x, w, (cos, sin) = chain_inputs(41, B=B, N=cap, H=H, d=d)
    q, k = binding.qk_norm_rope(x[:, :, :H], x[:, :, H:2 * H], *w, cos, sin)
    v = x[:, :, 2 * H:].transpose(1, 2).contiguous()
    kc, vc = torch.zeros_like(k), torch.zeros_like(v)
    kc[:, :, :N], vc[:, :, :N] = k[:, :, :N], v[:, :, :N]
    means = binding.block_means(kc, blk)
    for n in range(N, cap):
        pos = torch.full((B, 1), n, device="cuda", dtype=torch.int32)
        q1, k1 = binding.qk_norm_rope(x[:, n:n + 1, :H], x[:, n:n + 1, H:2 * H], *w, cos, sin,
                                      positions=pos)
        assert torch.equal(q1, q[:, :, n:n + 1]) and torch.equal(k1, k[:, :, n:n + 1])
        kc[:, :, n], vc[:, :, n] = k1[:, :, 0], v[:, :, n]
        if n % blk == 0:  # the block before this token's is complete
            means[:, :, n // blk - 1:n // blk] = binding.block_means(kc[:, :, n - blk:n], blk)
        if n % 37 and n + 1 < cap:
            continue
        ln = torch.tensor([n + 1], device="cuda", dtype=torch.int32)
        out, lse, blocks = binding.selected_decode(q1[:, :, 0].contiguous(), kc, vc, means, ln, 4, blk)
        for h in range(H):
            ro, rl, rb, eo, el = ops.selected_decode(
                f64(q[:, h, n]), f64(k[0, h]), f64(v[0, h]), ops.block_means(f64(k[0, h]), blk).astype(
                    np.float32).astype(np.float64), n + 1, 4, blk, d ** -0.5, U16)
            assert blocks[0, h].tolist() == rb
            check(out[:, h], ro, eo)
