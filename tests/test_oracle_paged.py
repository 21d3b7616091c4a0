"""Pins of the paged-cache oracle: closed forms and invariants that do not go through itself."""
import numpy as np
import pytest

import oracle
from oracle import paged as op


@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("R,d", [(8, 8), (4, 8)])
def test_rotation_keeps_lengths_and_depends_on_differences(style, R, d):
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 1, 1, d))
    th = op.scaled_thetas(100.0, R)
    turn = lambda a, p: op.norm_rope(a, None, 0.0, th, [p], style)  # noqa: E731
    assert np.isclose(np.linalg.norm(turn(x, 37)), np.linalg.norm(x))
    assert np.isclose((turn(x, 40) * turn(y, 33)).sum(), (turn(x, 7) * turn(y, 0)).sum())
    assert np.array_equal(turn(x, 5)[..., R:], x[..., R:])
    assert np.allclose(op.norm_rope(x, None, 0.0, th, [9], style, 1.5)[..., :R],
                       1.5 * turn(x, 9)[..., :R])


@pytest.mark.parametrize("style", ["half", "interleaved"])
def test_rotation_matches_the_shift_of_stored_keys(style):
    """Rotating to p, then shifting by s, is rotating to p + s."""
    rng = np.random.default_rng(2)
    k = rng.standard_normal((3, 2, 16))
    th = op.scaled_thetas(10000.0, 12)
    pos, shift = np.array([3, 50, 700]), np.array([-3, -20, -1])
    once = op.norm_rope(k, None, 0.0, th, pos, style)
    assert np.allclose(oracle.shift_keys(once, shift, 10000.0, 12, style),
                       op.norm_rope(k, None, 0.0, th, pos + shift, style))


def test_norm_closed_form():
    x = np.array([[[3.0, -4.0]]])
    got = op.norm_rope(x, np.array([1.0, 2.0]), 0.0, None, None, "half")
    assert np.allclose(got, [[[3.0 / np.sqrt(12.5), -8.0 / np.sqrt(12.5)]]])
    assert np.all(op.norm_rope(np.zeros((1, 1, 4)), np.ones(4), 1e-6, None, None, "half") == 0.0)


def test_scaled_frequencies():
    plain = op.scaled_thetas(10000.0, 8)
    assert np.allclose(plain, [1.0, 0.1, 0.01, 0.001])
    assert np.allclose(op.scaled_thetas(10000.0, 8, "linear", 4.0), plain / 4.0)
    base = op.scaled_thetas(10000.0, 8, "base", 4.0)      # the slowest pair is lowered by factor
    assert base[0] == 1.0 and np.isclose(base[-1], plain[-1] / 4.0)
    ramp = op.scaled_thetas(10000.0, 8, "ramp", 4.0, 2000.0, 1.0, 20.0)
    turns = 2000.0 * plain / (2 * np.pi)                  # 318, 31.8, 3.18, 0.318
    assert np.allclose(ramp[:2], plain[:2]) and np.isclose(ramp[3], plain[3] / 4.0)
    w = (turns[2] - 1.0) / 19.0
    assert np.isclose(ramp[2], plain[2] * (w + (1 - w) / 4.0))


def test_ragged_attention_over_shuffled_pages_is_chunk_attention():
    rng = np.random.default_rng(3)
    P, H, d = 4, 2, 8
    k, v = rng.standard_normal((2, 10, H, d))
    order = np.array([2, 0, 3])
    kp, vp = np.full((2, 5, P, H, d), np.nan)
    for r in range(10):
        kp[order[r // P], r % P], vp[order[r // P], r % P] = k[r], v[r]
    q = rng.standard_normal((4, 4, d))
    out, spread = op.ragged_attention(q, kp, vp, [order, order], [0, 3, 3], [10, 7], 0.3)
    assert np.allclose(out[:3], oracle.chunk_attention(q[:3], k, v, 0.3))
    assert np.isnan(out[3]).all() and (spread[:3] >= np.abs(out[:3])).all()
