"""Forms of the operators around the attention that only larger problems take, against the float64
reference: selections of more than 256 workgroups and their skip over tiles without candidates, gradients
whose lists are walked whole, and single tokens over long tables in one launch.  Bounds as in tests/test_gpu_operators.py."""

import numpy as np
import pytest

from oracle import operators as ops
from test_gpu_operators import U16, check, f64, gen, pack, randn, unpack

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------- selection ---

def runs(kind, rng, shape):
    """bool [..., n_qb, n_kb] whose rows have long runs without a bit."""
    n_qb, n_kb = shape[-2:]
    at = np.arange(n_kb)
    end = (np.arange(n_qb) + 1) * n_kb // n_qb
    if kind == "past":  # what lies before the row's end; nothing at all for the first rows
        on = np.broadcast_to(at < end[:, None] - 5, shape).copy()
    elif kind == "late":  # the first half is no row's
        on = np.broadcast_to(at >= n_kb // 2 + 3, shape).copy()
    else:  # "islands": a block here and there, tiles without any before, between and behind them
        on = rng.random(shape) < 0.5
        on &= (at // 16 % 5 == 2) | (at == n_kb - 1)
        on[..., n_qb // 2, :] = False
    return on


FORMS = [  # B, H, n_qb, n_kb, d, topk, candidates, keep
    (1, 40, 120, 100, 64, 9, None, None), (1, 40, 120, 100, 128, 17, None, "shared"),
    (2, 20, 120, 250, 128, 30, ("past", "shared"), None), (2, 20, 120, 250, 64, 30, ("late", "own"), "own"),
    (1, 40, 119, 591, 128, 59, ("past", "shared"), "shared"),
    (1, 40, 119, 591, 64, 20, ("islands", "shared"), None),
    (2, 20, 106, 1300, 128, 70, ("islands", "own"), "own"), (1, 40, 106, 1300, 64, 40, ("late", "shared"), None),
    (1, 2, 150, 11000, 64, 100, ("past", "shared"), None), (2, 1, 150, 11000, 128, 100, None, "shared"),
]


FEW = [(1, 2, 33, 591, 128, 59, ("past", "shared"), None), (2, 2, 17, 300, 64, 12, ("islands", "own"), None),
       (1, 3, 40, 1300, 128, 30, ("late", "own"), "shared"), (1, 1, 9, 6000, 64, 80, ("islands", "shared"), None)]


@pytest.mark.parametrize("many,case", [(True, c) for c in FORMS] + [(False, c) for c in FEW])
def test_block_select_forms(many, case):
    import torch
    from paper_2606_23019_amd import binding
    B, H, n_qb, n_kb, d, topk, cand, keep = case
    together = min(16, 156 * 1024 // (-(-n_kb // 16) * 16 * 8))
    assert (B * H * -(-n_qb // together) > 256) == many  # the form's line
    g = gen(n_kb + d)
    qm, km = (torch.randn((B, H, n, d), generator=g, device="cuda") for n in (n_qb, n_kb))
    km[:, :, n_kb // 2:] = km[:, :, :n_kb - n_kb // 2].clone()  # every score twice
    rng = np.random.default_rng(n_kb)
    con = kon = None
    if cand:
        con = runs(cand[0], rng, (B if cand[1] == "own" else 1, H, n_qb, n_kb))
    if keep:
        kon = rng.random((B if keep == "own" else 1, H, n_qb, n_kb)) < 0.02
    bits = lambda on, kind: None if on is None else pack(on if kind == "own" else on[0])
    mask = binding.block_select(qm, km, topk, candidates=bits(con, cand and cand[1]), keep=bits(kon, keep))
    got = unpack(mask, n_kb)
    for b in range(B):
        for h in sorted({0, H // 3, H - 1}):
            one = lambda on: None if on is None else on[b % len(on), h]
            ref = ops.block_select(f64(qm[b, h]), f64(km[b, h]), topk, one(con), one(kon))
            assert np.array_equal(got[b, h], ref), (b, h, np.argwhere(got[b, h] != ref)[:4])
    # the other heads: as many blocks as there have to be
    n = np.full((B, H, n_qb), min(topk, n_kb)) if con is None else np.minimum(con.sum(-1), topk)
    assert (got.sum(-1) >= n).all() and (keep or (got.sum(-1) == n).all())


# --------------------------------------------------------------- gradients ---

WHOLE = [  # B, H, N, d, blk_q, blk_k, layout, a mask for every batch entry
    (1, 40, 1500, 64, 64, 64, "bhnd", False), (1, 40, 1530, 128, 64, 64, "bnhd", False),
    (2, 20, 3000, 128, 128, 128, "bhnd", True), (1, 40, 3001, 64, 128, 128, "bnhd", False),
    (2, 24, 2990, 128, 128, 64, "bhnd", False), (1, 48, 2990, 64, 128, 64, "bhnd", False),
    (2, 24, 3050, 128, 64, 128, "bnhd", True), (1, 48, 3050, 64, 64, 128, "bhnd", False),
]


@pytest.mark.parametrize("case", WHOLE)
def test_bsattn_bwd_of_whole_lists(case):
    """More than 1024 pairs of blocks in all: lists up to a 512th of them are walked by one
    workgroup, longer ones (a row that sees all, a column that all see) are cut and joined."""
    import torch
    from paper_2606_23019_amd import binding
    B, H, N, d, blk_q, blk_k, layout, own = case
    g = gen(N + d)
    shape = (B, H, N, d) if layout == "bhnd" else (B, N, H, d)
    q, k, v, dout = (randn(g, *shape) for _ in range(4))
    n_qb, n_kb = -(-N // blk_q), -(-N // blk_k)
    rng = np.random.default_rng(N + d)
    # few blocks in most heads, so that the lists of others are long beside a 512th of all
    rho = np.where(np.arange(H) % 8 == 3, 0.55, rng.uniform(0.05, 0.4, H))
    on = rng.random((B if own else 1, H, n_qb, n_kb)) < rho[None, :, None, None]
    on[:, 0::5, n_qb - 2] = True
    on[:, 0::5, :, n_kb // 3] = True
    on[:, 1::5, 2] = False
    on[:, :, n_qb - 1, n_kb - 1] = True  # the ragged corner
    total = on.sum() * (1 if own else B)
    limit = max(2, -(-total // 512))
    sides = [on.sum(axis) for axis in (-1, -2)]
    for lists in sides:
        assert ((lists > 2) & (lists <= limit)).sum() > lists.size // 2 and lists[lists <= limit].max() >= 8
    cut = [(lists > limit).any() for lists in sides]
    assert all(cut) if blk_q == blk_k else any(cut)
    heads = (lambda t: t) if layout == "bhnd" else (lambda t: t.transpose(1, 2))
    out, lse = torch.empty_like(q), torch.empty((B, H, N), device="cuda")
    for b in range(B):  # the forward call has one mask for all of its batch entries
        fwd = binding.bsattn_fwd if layout == "bhnd" else binding.bsattn_fwd_bnhd
        o, l = fwd(*(t[b:b + 1].contiguous() for t in (q, k, v)), pack(on[b if own else 0]), blk_q, blk_k)
        out[b], lse[b] = o[0], l[0]
    mask = pack(on if own else on[0])
    got = binding.bsattn_bwd(dout, q, k, v, out, lse, mask, blk_q, blk_k, layout=layout)
    again = binding.bsattn_bwd(dout, q, k, v, out, lse, mask, blk_q, blk_k, layout=layout)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for b, h in ((0, 0), (B - 1, 3), (B - 1, H - 4)):
        see = on[b if own else 0, h].repeat(blk_q, 0)[:N].repeat(blk_k, 1)[:, :N]
        x = [f64(heads(t)[b, h]) for t in (dout, q, k, v, out)]
        ref, bound = ops.attention_grad(*x, f64(lse[b, h]), see, d ** -0.5, U16)
        for t, r, e in zip(got, ref, bound):
            check(heads(t)[b, h], r, e)


# ------------------------------------------------------------ single tokens ---

LONG = [  # B, Hq, Hkv, cap, d, blk, topk, lengths: up to 64 units of 32 keys, 2048 blocks
    (2, 2, 1, 131072, 128, 64, 32, [131072, 100001]), (1, 2, 2, 262140, 128, 128, 16, [262100]),
    (2, 17, 1, 90001, 128, 64, 20, [90001, 81930]), (1, 1, 1, 131072, 64, 64, 32, [131071]),
    (2, 4, 4, 40000, 128, 64, 9, [40000, 20000]), (3, 8, 2, 20000, 128, 64, 32, [20000, 16400, 2100]),
    (1, 3, 1, 70000, 128, 128, 16, [69999]),
]


@pytest.mark.parametrize("case", LONG)
def test_decode_in_one_launch_over_long_tables(case):
    import torch
    from paper_2606_23019_amd import binding
    B, Hq, Hkv, cap, d, blk, topk, lengths = case
    assert topk * blk // 32 <= 64 and -(-cap // blk) <= 2048  # the form's lines
    g = gen(cap)
    q, k, v = randn(g, B, Hq, d), randn(g, B, Hkv, cap, d), randn(g, B, Hkv, cap, d)
    means = binding.block_means(k, blk)
    for b, n in enumerate(lengths):  # nothing past the last token is read
        k[b, :, n:], v[b, :, n:] = float("nan"), float("nan")
        means[b, :, -(-n // blk) - 1:] = float("nan")
    ln = torch.tensor(lengths, device="cuda", dtype=torch.int32)
    out, lse, blocks = binding.selected_decode(q, k, v, means, ln, topk, blk)
    G = Hq // Hkv
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            rows = slice(h * G, (h + 1) * G)
            ro, rl, rb, eo, el = ops.selected_decode(f64(q[b, rows]), f64(k[b, h]), f64(v[b, h]),
                                                     f64(means[b, h]), n, topk, blk, d ** -0.5, U16)
            assert blocks[b, h].tolist() == rb + [-1] * (topk - len(rb))
            check(out[b, rows], ro, eo)
            assert (np.abs(f64(lse[b, rows]) - rl) <= el).all()


def test_decode_of_the_largest_topk():
    """topk of 2^31 - 1 over a table of two blocks: the list is filled to its end, and what lies
    around it stays as it was."""
    import ctypes
    import torch
    from paper_2606_23019_amd import binding
    P, topk, pad = ctypes.c_void_p, (1 << 31) - 1, 4096
    g = gen(3)
    q, k, v = randn(g, 1, 2, 64), randn(g, 1, 1, 100, 64), randn(g, 1, 1, 100, 64)
    means = binding.block_means(k, 64)
    ln = torch.tensor([99], device="cuda", dtype=torch.int32)
    out, lse = torch.empty_like(q), torch.empty((1, 2), device="cuda")
    room = torch.full((topk + 2 * pad,), 7, device="cuda", dtype=torch.int32)
    blocks = room[pad:-pad]
    lib = binding.load()
    n = lib.sa_selected_decode_workspace(1, 2, 1, 100, 64, 64, topk)
    ws = torch.empty(max(n, 1), device="cuda", dtype=torch.uint8)
    strides = (ctypes.c_int64 * 3)(0, 0, 64)
    assert lib.sa_selected_decode(P(q.data_ptr()), P(k.data_ptr()), P(v.data_ptr()), strides, P(means.data_ptr()),
                                  P(ln.data_ptr()), P(out.data_ptr()), P(lse.data_ptr()), P(blocks.data_ptr()),
                                  P(ws.data_ptr()), 1, 2, 1, 100, 64, 64, topk, 0.125, binding._stream(None)) == 0
    torch.cuda.synchronize()
    ro, rl, rb, eo, el = ops.selected_decode(f64(q[0]), f64(k[0, 0]), f64(v[0, 0]), f64(means[0, 0]), 99,
                                             2, 64, 0.125, U16)
    assert blocks[:2].tolist() == rb and bool((blocks[2:] == -1).all())
    assert bool((room[:pad] == 7).all()) and bool((room[-pad:] == 7).all())
    check(out[0], ro, eo)
    assert (np.abs(f64(lse[0]) - rl) <= el).all()
