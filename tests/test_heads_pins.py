"""The oracle of the head operators against the other oracle, against differences, and against what rotations are (CPU)."""
import numpy as np
import pytest

from oracle import heads as oh
from oracle import rope as orope


def _angles(rng, rows, rot):
    a = rng.uniform(-3, 3, (rows, rot // 2))
    return np.cos(a), np.sin(a)


def test_half_layout_is_the_projections_rotation():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 6 * 16))           # two query heads, two key heads, two of v
    cos, sin = _angles(rng, 9, 16)
    pos = np.array([8, 0, 3, 3, 1])
    want = orope.rope_rows(x, pos, cos, sin, 2, 2, 16)
    got = oh.turn(x.reshape(5, 6, 16)[:, :4], cos[pos], sin[pos], False)
    assert np.allclose(got.reshape(5, -1), want[:, :64], atol=1e-15) and np.array_equal(want[:, 64:], x[:, 64:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations_add_up_and_keep_lengths(interleaved):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((4, 3, 20))
    a, b = rng.uniform(-3, 3, (2, 4, 6))
    once = oh.turn(oh.turn(x, np.cos(a), np.sin(a), interleaved), np.cos(b), np.sin(b), interleaved)
    assert np.allclose(once, oh.turn(x, np.cos(a + b), np.sin(a + b), interleaved), atol=1e-14)
    assert np.allclose((once ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(once[..., 12:], x[..., 12:])


def test_layouts_are_a_permutation_apart():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 3, 12))
    c, s = _angles(rng, 4, 8)
    order = np.array([0, 4, 1, 5, 2, 6, 3, 7, 8, 9, 10, 11])      # halves -> neighbours
    assert np.allclose(oh.turn(x[..., order], c, s, True), oh.turn(x, c, s, False)[..., order], atol=1e-15)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rot", [0, 8, 12])
def test_gradients_are_differences(interleaved, norm, rot):
    rng = np.random.default_rng(4)
    x, g, w = rng.standard_normal((3, 2, 12)), rng.standard_normal((3, 2, 12)), rng.uniform(0.5, 1.5, 12) if norm else None
    c, s = _angles(rng, 3, rot) if rot else (None, None)
    dx, dxs, dw, dws = oh.heads_back(x, g, w, 1e-3, c, s, interleaved)
    f = lambda x, w: (oh.heads(x, w, 1e-3, c, s, interleaved)[0] * g).sum()
    h = 1e-6
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[at]) < 1e-8
        assert abs(dx[at]) <= dxs[at] + 1e-15
    for i in range(12 if norm else 0):
        e = np.zeros(12)
        e[i] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[i]) < 1e-8 and abs(dw[i]) <= dws[i] + 1e-15


def test_scaled_tables():
    c, s = oh.tables(8, 10000.0, 5, 3)
    assert np.allclose(c[:, 0], np.cos([5, 6, 7])) and np.allclose(s[:, 2], np.sin(np.array([5, 6, 7]) / 100))
    lc, _ = oh.tables(8, 10000.0, 20, 12, "linear", 4.0)
    assert np.allclose(lc[::4], c)                                  # position 4 p is what position p was
    # by parts: pair 0 turns 1000 / 2 pi = 159 times in the original positions, pair 3 0.16 times
    pc, ps = oh.tables(8, 10000.0, 0, 50, "by_parts", 4.0, original=1000, low=1, high=32, magnitude=2.0)
    pl, lin = oh.tables(8, 10000.0, 0, 50)[0], oh.tables(8, 10000.0, 0, 50, "linear", 4.0)[0]
    assert np.allclose(pc[:, 0], 2 * pl[:, 0]) and np.allclose(pc[:, 3], 2 * lin[:, 3])
    g = (1000 * 0.1 / (2 * np.pi) - 1) / 31
    assert np.allclose(ps[:, 1], 2 * np.sin(np.arange(50) * 0.1 * (g + (1 - g) / 4)))
    big, _ = oh.tables(4, 1e6, 2 ** 24 - 1, 1)
    assert abs(float(big[0, 0]) - np.cos(float(2 ** 24 - 1))) < 1e-9
