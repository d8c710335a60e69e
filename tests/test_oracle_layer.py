"""The oracle of norm, rotation and windowed attention against what can be said without it: lengths kept, relative positions, plain attention
as the special case, and gradients against differences."""
import numpy as np
import pytest

from oracle import layer_oracle as L

ROPE = [((16, 24, 24), True), ((64,), False), ((32,), False), ((16, 32), False), ((2,), True)]


@pytest.mark.parametrize("dims,interleaved", ROPE)
def test_rotation_keeps_lengths_and_sees_relative_positions(dims, interleaved):
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(2, 5, 64))
    pos = rng.integers(0, 1000, (5, len(dims)))
    turn = lambda z, p: L.qk_norm_rope(z, p, dims, 1e4, interleaved, np.ones(64), 0.0)  # noqa: E731
    a = turn(x, pos)
    np.testing.assert_allclose((a * a).mean(-1), 1.0, rtol=1e-12)
    np.testing.assert_allclose((a * turn(y, pos)).sum(-1), (turn(x, pos + 77) * turn(y, pos + 77)).sum(-1), atol=1e-9)
    np.testing.assert_allclose(turn(x, 0 * pos), x / np.sqrt((x * x).mean(-1, keepdims=True)), rtol=1e-12)
    assert (turn(x, pos)[:, sum(dims):] == turn(x, 0 * pos)[:, sum(dims):]).all()


def test_rotation_of_one_pair_by_hand():
    out = L.qk_norm_rope(np.array([[3.0, 4.0]]), np.array([[2]]), (2,), 1e4, True, np.ones(2), 0.0)
    a, b = np.array([3.0, 4.0]) / np.sqrt(12.5)
    np.testing.assert_allclose(out[0], [a * np.cos(2) - b * np.sin(2), a * np.sin(2) + b * np.cos(2)], rtol=1e-12)


@pytest.mark.parametrize("dims,interleaved", ROPE)
def test_rope_gradients_against_differences(dims, interleaved):
    rng = np.random.default_rng(2)
    x, up = rng.normal(size=(2, 3, 64))
    w, pos = 1 + 0.3 * rng.normal(size=64), rng.integers(0, 50, (3, len(dims)))
    f = lambda x_, w_: (L.qk_norm_rope(x_, pos, dims, 1e4, interleaved, w_, 1e-3) * up).sum()  # noqa: E731
    dx, dw = L.qk_norm_rope_bwd(x, up, pos, dims, 1e4, interleaved, w, 1e-3)
    e = 1e-5
    for _ in range(20):
        ex, ew = rng.normal(size=x.shape), rng.normal(size=64)
        np.testing.assert_allclose((f(x + e * ex, w) - f(x - e * ex, w)) / (2 * e), (dx * ex).sum(), rtol=1e-6, atol=1e-7)
        np.testing.assert_allclose((f(x, w + e * ew) - f(x, w - e * ew)) / (2 * e), (dw * ew).sum(), rtol=1e-6, atol=1e-7)


def test_window_mask_by_hand():
    see = L.window_mask(3, 6, 1, 0, 1).astype(int)
    assert see.tolist() == [[1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert L.window_mask(3, 2, -1, 0, 5).astype(int).tolist() == [[0, 0], [1, 0], [1, 1]]           # the first row is in front of every key
    assert L.window_mask(2, 4, 0, 1, 0).astype(int).tolist() == [[0, 0, 1, 1], [0, 0, 0, 1]]
    assert L.window_mask(4, 4, -1, -1, 0).all()


def test_no_limits_is_plain_attention():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 7, 8))
    s = np.exp(q @ k.T / np.sqrt(8))
    o, lse, _ = L.window_attn(q, k, v, L.window_mask(7, 7, -1, -1, 0), 1 / np.sqrt(8))
    np.testing.assert_allclose(o, s @ v / s.sum(-1, keepdims=True), rtol=1e-12)
    np.testing.assert_allclose(lse, np.log(s.sum(-1)), rtol=1e-12)


@pytest.mark.parametrize("n_q,n_k,left,right,sinks", [(9, 9, 2, 0, 1), (5, 8, 1, 2, 2), (6, 4, -1, 0, 0), (4, 4, 0, 0, 0)])
def test_window_gradients_against_differences(n_q, n_k, left, right, sinks):
    rng = np.random.default_rng(4)
    see = L.window_mask(n_q, n_k, left, right, sinks)
    x = [rng.normal(size=(n, 8)) for n in (n_q, n_k, n_k)]
    d_o = rng.normal(size=(n_q, 8))
    f = lambda y: (L.window_attn(*y, see, 0.4)[0] * d_o).sum()  # noqa: E731
    grads, e = L.window_attn_bwd(*x, see, 0.4, d_o), 1e-5
    for _ in range(20):
        for i in range(3):
            step = rng.normal(size=x[i].shape)
            up, down = ([y + s * e * step if j == i else y for j, y in enumerate(x)] for s in (1, -1))
            np.testing.assert_allclose((f(up) - f(down)) / (2 * e), (grads[i] * step).sum(), rtol=1e-6, atol=1e-7)
