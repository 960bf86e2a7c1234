"""Reference of the operators around the attention, float64 on the CPU.

Test infrastructure only (see ``oracle/__init__``).  Plain NumPy from the
definitions, one head at a time where a head is large:

  norm_rope, norm_rope_grad   RMS norm of every head's rows and the rotation by
                              position, and the gradients of a loss through it
  block_means, block_select   means of blocks of tokens; the best key blocks of
                              each query block by the products of means
  attention_grad              gradients of softmax attention over the pairs of a
                              boolean mask, with out and lse as the forward pass
                              left them
  selected_decode             one query token a sequence over selected blocks

``attention_grad`` and ``selected_decode`` return, beside the values, what the
values can be off by when probabilities and score gradients are rounded to
``u_p`` relative and every sum runs in fp32 in any order.
"""

import numpy as np

U32 = 2.0 ** -24  # half a step of fp32, relative


def turn(x, cos, sin, pairs, sign=1.0):
    """x [..., d] with its first 2 cos.shape[-1] elements turned pair by pair."""
    half = cos.shape[-1]
    y = np.array(x, dtype=np.float64)
    if pairs == "interleaved":
        i, j = np.arange(half) * 2, np.arange(half) * 2 + 1
    else:
        i, j = np.arange(half), np.arange(half) + half
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i] = a * cos - sign * b * sin
    y[..., j] = b * cos + sign * a * sin
    return y


def norm_rope(x, w, cos, sin, eps, pairs):
    """x [B, N, H, d]; cos, sin [B, N, rot / 2]: [B, N, H, d]."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return turn(x * r * w, cos[:, :, None], sin[:, :, None], pairs)


def norm_rope_grad(dy, x, w, cos, sin, eps, pairs):
    """(dx, dw) of sum(dy * norm_rope(x, w))."""
    g = turn(dy, cos[:, :, None], sin[:, :, None], pairs, -1.0)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    dx = r * (g * w - n * (g * w * n).mean(-1, keepdims=True))
    return dx, (g * n).sum((0, 1, 2))


def block_means(x, blk):
    """[..., N, d] -> [..., ceil(N / blk), d]."""
    N = x.shape[-2]
    return np.stack([x[..., i:i + blk, :].mean(-2) for i in range(0, N, blk)], -2)


def best(score, may, topk):
    """Places of the topk largest scores among ``may``, ties to the lowest place."""
    at = [v for v in range(len(score)) if may[v]]
    at.sort(key=lambda v: (-score[v] if score[v] == score[v] else np.inf,
                           score[v] != score[v], v))
    return sorted(at[:topk])


def block_select(qm, km, topk, candidates=None, keep=None):
    """bool [n_qb, n_kb] of one head from its means (float64 of the fp32 ones)."""
    n_qb, n_kb = len(qm), len(km)
    on = np.zeros((n_qb, n_kb), dtype=bool)
    for u in range(n_qb):
        with np.errstate(invalid="ignore", over="ignore"):
            score = (km * qm[u]).sum(-1)
        on[u, best(score, np.ones(n_kb, bool) if candidates is None else candidates[u], topk)] = True
        if keep is not None:
            on[u] |= keep[u]
    return on


def _score_error(q, k, scale, d):
    """What scale * <q, k> in fp32 can be off by, for every pair."""
    return (d + 8) * U32 * scale * (np.abs(q) @ np.abs(k).T)


def attention_grad(dout, q, k, v, out, lse, see, scale, u_p):
    """((dq, dk, dv), (their bounds)) of one head; see: bool [N, N] pairs of the mask."""
    d = q.shape[1]
    s = scale * (q @ k.T)
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(see, np.exp(s - lse[:, None]), 0.0)
    dp = dout @ v.T
    delta = (dout * out).sum(1, keepdims=True)
    ds = p * (dp - delta)
    values = (scale * (ds @ k), scale * (ds.T @ q), p.T @ dout)
    # relative error of p: of its exponent (the product, and lse and the scale folded into
    # it) and of exp itself
    lse0 = np.where(np.isfinite(lse), lse, 0.0)
    rel = _score_error(q, k, scale, d) + 8 * U32 * (np.abs(lse0)[:, None] + np.abs(s)) + 2.0 ** -20
    a, g = np.abs(dout), np.abs(p)
    inner = (d + 8) * U32 * (a @ np.abs(v).T + (a * np.abs(out)).sum(1, keepdims=True))
    e_p = g * (rel + u_p)
    e_ds = np.abs(ds) * (rel + u_p) + g * inner * (1 + u_p)
    n = q.shape[0] * U32 + 4 * U32  # the sums over the pairs, in any order
    bounds = (scale * ((e_ds + n * np.abs(ds)) @ np.abs(k)),
              scale * ((e_ds + n * np.abs(ds)).T @ np.abs(q)), (e_p + n * g).T @ a)
    return values, bounds


def selected_decode(q, k, v, means, length, topk, blk, scale, u_p):
    """One sequence and one key head: q [G, d], k and v [cap, d], means [n, d].

    Returns (out, lse, blocks, bound of out, bound of lse)."""
    G, d = q.shape
    if length == 0:
        return np.zeros((G, d)), np.full(G, -np.inf), [], np.zeros((G, d)), np.zeros(G)
    last = (length + blk - 1) // blk - 1
    score = (means[:last] * q.sum(0)).sum(-1)
    blocks = best(score, np.ones(last, bool), topk - 1) + [last]
    rows = np.concatenate([np.arange(b * blk, min((b + 1) * blk, length)) for b in blocks])
    s = scale * (q @ k[rows].T)
    top = s.max(1, keepdims=True)
    total = np.exp(s - top).sum(1, keepdims=True)
    lse = (top + np.log(total))[:, 0]
    p = np.exp(s - lse[:, None])
    out = p @ v[rows]
    # a probability is off by its exponent's error, twice (its own and the sum's), by its
    # rounding, and by the sums' rounding
    rel = (_score_error(q, k[rows], scale, d) + 8 * U32 * np.abs(s) + 2.0 ** -20).max(1, keepdims=True)
    rel = 2 * rel + u_p + (len(rows) + 64) * U32
    return (out, lse, blocks, rel * (p @ np.abs(v[rows])),
            rel[:, 0] - u_p + 8 * U32 * np.abs(lse) + 2.0 ** -20)
