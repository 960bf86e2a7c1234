"""The reference of the operators around the attention against differences and hand-made cases."""

import numpy as np
import pytest

from oracle import operators as ops


def _difference(loss, x, h=1e-5):
    g = np.zeros_like(x)
    flat = x.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + h
        up = loss()
        flat[i] = keep - h
        down = loss()
        flat[i] = keep
        g.reshape(-1)[i] = (up - down) / (2 * h)
    return g


# A central difference with h = 1e-5 of a loss of size L is off by L'' h^2 and by the
# rounding 2^-53 |L| / h: 1e-8 and less here.
TOL = 1e-6


@pytest.mark.parametrize("pairs,rot", [("interleaved", 8), ("halves", 8), ("halves", 4)])
def test_norm_rope_gradient_is_the_difference(pairs, rot):
    rng = np.random.default_rng(3)
    B, N, H, d = 2, 3, 2, 8
    x, dy = rng.standard_normal((2, B, N, H, d))
    w = 1 + 0.2 * rng.standard_normal(d)
    angle = rng.uniform(-3, 3, (B, N, rot // 2))
    cos, sin = np.cos(angle), np.sin(angle)

    def loss():
        return (dy * ops.norm_rope(x, w, cos, sin, 1e-3, pairs)).sum()
    dx, dw = ops.norm_rope_grad(dy, x, w, cos, sin, 1e-3, pairs)
    assert np.abs(dx - _difference(loss, x)).max() < TOL
    assert np.abs(dw - _difference(loss, w)).max() < TOL


def test_norm_rope_by_hand():
    x = np.array([3.0, 4.0, 0.0, 0.0]).reshape(1, 1, 1, 4)
    quarter = np.zeros((1, 1, 1)), np.ones((1, 1, 1))  # cos, sin of a right angle
    r = 1 / np.sqrt(25 / 4)
    got = ops.norm_rope(x, np.ones(4), *quarter, 0.0, "interleaved")[0, 0, 0]
    assert np.allclose(got, [-4 * r, 3 * r, 0, 0])
    got = ops.norm_rope(x, np.ones(4), *quarter, 0.0, "halves")[0, 0, 0]
    assert np.allclose(got, [-4 * r, 3 * r, 0, 0])  # rot = 2: elements 0 and 1
    wide = np.zeros((1, 1, 2)), np.ones((1, 1, 2))
    got = ops.norm_rope(x, np.ones(4), *wide, 0.0, "halves")[0, 0, 0]
    assert np.allclose(got, [0, 0, 3 * r, 4 * r])


def test_attention_gradient_is_the_difference():
    rng = np.random.default_rng(4)
    N, d, scale = 7, 4, 0.6
    q, k, v, dout = rng.standard_normal((4, N, d))
    see = rng.random((N, N)) < 0.5
    see[2] = False  # a row with nothing
    see[:, 5] = False  # a key that no row sees

    def forward():
        s = np.where(see, scale * (q @ k.T), -np.inf)
        with np.errstate(divide="ignore"):
            lse = np.log(np.exp(s).sum(1))
        p = np.where(see, np.exp(s - np.where(np.isinf(lse), 0, lse)[:, None]), 0.0)
        return p @ v, lse

    def loss():
        return (dout * forward()[0]).sum()
    out, lse = forward()
    got, _ = ops.attention_grad(dout, q, k, v, out, lse, see, scale, 0.0)
    for g, x in zip(got, (q, k, v)):
        assert np.abs(g - _difference(loss, x)).max() < TOL
    assert not got[0][2].any() and not got[1][5].any() and not got[2][5].any()


def test_best_takes_ties_by_place_and_nan_last():
    nan = np.nan
    assert ops.best(np.array([1.0, 3, 3, 2, 3]), np.ones(5, bool), 2) == [1, 2]
    assert ops.best(np.array([nan, -np.inf, 0, 1]), np.ones(4, bool), 3) == [1, 2, 3]
    assert ops.best(np.array([5.0, 1, 4]), np.array([False, True, True]), 9) == [1, 2]


def test_block_means_and_select_by_hand():
    x = np.arange(10.0).reshape(5, 2)
    assert np.array_equal(ops.block_means(x, 2), [[1, 2], [5, 6], [8, 9]])
    on = ops.block_select(np.array([[1.0], [-1.0]]), np.array([[1.0], [2.0], [2.0]]), 1,
                          keep=np.array([[True, False, False], [False, False, False]]))
    assert np.array_equal(on, [[True, True, False], [True, False, False]])


def test_decode_is_attention_over_everything_when_all_blocks_are_taken():
    rng = np.random.default_rng(5)
    q = rng.standard_normal((2, 4))
    k, v = rng.standard_normal((2, 12, 4))
    out, lse, blocks, _, _ = ops.selected_decode(q, k, v, ops.block_means(k, 4), 10, 9, 4, 0.5, 0.0)
    s = np.exp(0.5 * (q @ k[:10].T))
    assert blocks == [0, 1, 2]
    assert np.allclose(out, (s / s.sum(1, keepdims=True)) @ v[:10]) and np.allclose(lse, np.log(s.sum(1)))
