"""The oracle of the norm and rotation, pinned by closed forms and invariants."""
import numpy as np
import pytest

from oracle.qkv import norm_rope, rope_table


def _x(T=5, h=2, d=64, seed=0):
    return np.random.default_rng(seed).standard_normal((T, h, d))


def test_norm_gives_unit_mean_square_times_the_weight():
    w = np.linspace(0.5, 2, 64)
    y, _ = norm_rope(_x(), weight=w)
    assert np.allclose(((y / w) ** 2).mean(-1), 1)
    z, _ = norm_rope(1000 * _x(), weight=w)
    assert np.allclose(y, z)


def test_norm_by_hand():
    y, size = norm_rope(np.array([[[3.0, 4.0]]]), weight=[2.0, 1.0], eps=11.5)
    assert np.allclose(y, [[[3 * 2 / np.sqrt(24), 4 / np.sqrt(24)]]])
    assert np.allclose(size, np.abs(y))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_the_rest(interleaved):
    x, t = _x(d=64), rope_table(100, 32)
    y, _ = norm_rope(x, table=t, positions=[0, 7, 99, 3, 3], interleaved=interleaved)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-6)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose(y[0], x[0])                      # position 0
    assert np.allclose(y[4], norm_rope(x[4:], table=t, positions=[3],
                                       interleaved=interleaved)[0][0])


def test_rotation_by_hand():
    t = np.array([[np.cos(0.3), np.cos(0.5), np.sin(0.3), np.sin(0.5)]], np.float64)
    x = np.array([[[1.0, 0.0, 0.0, 2.0]]])
    y, _ = norm_rope(x, table=t, positions=[0])         # pairs (0, 2), (1, 3)
    assert np.allclose(y, [[[np.cos(0.3), -2 * np.sin(0.5), np.sin(0.3), 2 * np.cos(0.5)]]])
    y, _ = norm_rope(x, table=t, positions=[0], interleaved=True)
    assert np.allclose(y, [[[np.cos(0.3), np.sin(0.3), -2 * np.sin(0.5), 2 * np.cos(0.5)]]])


@pytest.mark.parametrize("interleaved", [False, True])
def test_dot_products_depend_on_the_distance_alone(interleaved):
    q, k = _x(1, 1, 64, 1), _x(1, 1, 64, 2)
    t = rope_table(3000, 64).astype(np.float64)

    def dot(p, s):
        return float((norm_rope(q, table=t, positions=[p], interleaved=interleaved)[0] *
                      norm_rope(k, table=t, positions=[s], interleaved=interleaved)[0]).sum())
    assert dot(17, 5) == pytest.approx(dot(2012, 2000), abs=1e-4)
    assert abs(dot(17, 5) - dot(17, 6)) > 1e-3


def test_axes():
    x, t = _x(4), rope_table(50, 64)
    same = np.tile([3, 1, 49, 0], (3, 1))
    one, _ = norm_rope(x, table=t, positions=same[0])
    assert np.array_equal(norm_rope(x, table=t, positions=same, sections=(5, 20, 7))[0], one)
    pos = np.array([[1, 2, 3, 4], [0, 0, 0, 0], [9, 9, 9, 9]])
    y, _ = norm_rope(x, table=t, positions=pos, sections=(5, 20, 7))
    for axis, dims in ((0, range(0, 5)), (1, range(5, 25)), (2, range(25, 32))):
        alone, _ = norm_rope(x, table=t, positions=pos[axis])
        for i in dims:
            assert np.array_equal(y[..., [i, i + 32]], alone[..., [i, i + 32]])
    assert np.allclose(y[..., 5:25], x[..., 5:25])


def test_positions_outside_the_table_are_nan():
    y, _ = norm_rope(_x(3), table=rope_table(10, 32), positions=[-1, 10, 9])
    assert np.isnan(y[:2, :, :32]).all() and np.isfinite(y[2]).all()
    assert np.isfinite(y[..., 32:]).all()
