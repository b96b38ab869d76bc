"""Pins of the packed sequences' oracle (oracle/packed.py): closed forms and the identities that define it."""

import math

import numpy as np
import pytest

from oracle import attention, packed, rope


def test_plain_frequencies_and_rotation_are_the_full_rotary():
    theta = packed.frequencies(64, 10000.0)
    assert np.allclose(theta, rope.inv_freq(64, 10000.0), rtol=1e-14)
    x = np.random.default_rng(0).standard_normal((5, 3, 64))
    pos = np.array([0, 1, 77, -5, 100000])
    for pairing in ("half", "interleaved"):
        assert np.allclose(packed.rotate(x, pos, theta, pairing), rope.rotate(x, pos, 10000.0, pairing), atol=1e-9)


def test_partial_rotation_leaves_the_rest_and_pairs_inside_the_part():
    x = np.random.default_rng(1).standard_normal((4, 2, 128))
    theta = packed.frequencies(32, 500.0)
    y = packed.rotate(x, np.arange(4), theta, "half", amplitude=1.5)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose(np.hypot(y[..., :16], y[..., 16:32]), 1.5 * np.hypot(x[..., :16], x[..., 16:32]), rtol=1e-13)


def test_scalings_at_their_ends():
    dim, base, s, L = 64, 10000.0, 8.0, 4096.0
    plain = packed.frequencies(dim, base)
    assert np.allclose(packed.frequencies(dim, base, "linear", s), plain / s)
    by_base = packed.frequencies(dim, base, "base", s)
    assert by_base[0] == 1.0 and math.isclose(by_base[-1], plain[-1] / s, rel_tol=1e-12)   # slowest: interpolated
    turns = L * plain / (2 * math.pi)
    rot = packed.frequencies(dim, base, "rotations", s, L, 32.0, 1.0)
    assert np.allclose(rot[turns >= 32], plain[turns >= 32]) and np.allclose(rot[turns <= 1], plain[turns <= 1] / s)
    assert np.all((rot <= plain) & (rot >= plain / s * (1 - 1e-12)))
    idx = packed.frequencies(dim, base, "index", s, L, 32.0, 1.0)
    # 32 / ln(1e4) ln(4096 / 2 pi n) = 10.47 for 32 turns, 22.5 for one: lo = 10, hi = 23
    assert np.allclose(idx[:11], plain[:11]) and np.allclose(idx[23:], plain[23:] / s)
    assert math.isclose(idx[14], plain[14] * (9 / 13) + plain[14] / s * (4 / 13), rel_tol=1e-12)


def test_rms_norm():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    y = packed.rms_norm(x, np.array([0.0, 1.0, 0.0, 0.0]), 0.0, 1.0)
    assert np.allclose(y, [[3 / 2.5, 2 * 4 / 2.5, 0, 0]])
    assert np.array_equal(packed.rms_norm(np.zeros((1, 4)), np.ones(4), 1e-6, 0.0), np.zeros((1, 4)))


@pytest.mark.parametrize("window", [0, 7])
def test_attention_is_the_oracle_attention(window):
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((6, 4, 16)), rng.standard_normal((30, 2, 16)), rng.standard_normal((30, 2, 16))
    index = np.array([0, 3, 8, 9, 20, 29])
    out, spread, mass, _ = packed.attend_bounds(q, index, k, v, 0.25, window)
    assert np.allclose(out, attention.attend(q, index, k, v, 0.25, window), atol=1e-12)
    assert np.all(spread[0] == 0) and np.allclose(mass[0], np.abs(np.repeat(v[0], 2, axis=0)))   # one key
    assert np.all(spread <= mass + np.abs(out) + 1e-12)
