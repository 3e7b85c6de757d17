"""Pins of the decoding oracle: rotations against complex multiplication and known values, attention against hand-built
cases, gradients against differences."""
import math

import numpy as np
import pytest

from oracle import decode


def test_rotation_by_hand():
    # one pair, frequency 1: a quarter turn maps (1, 0) to (0, 1); the rest of the row is copied
    x = np.array([[[1.0, 0.0, 7.0]]])
    y = decode.rotate(x, [1], [math.pi / 2])
    assert np.allclose(y, [[[0.0, 1.0, 7.0]]])
    assert np.allclose(decode.rotate(y, [1], [math.pi / 2], inverse=True), x)
    # halves and neighbours pair differently
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    half = decode.rotate(x, [2], [math.pi / 4, 0.0])
    assert np.allclose(half, [[[-3.0, 2.0, 1.0, 4.0]]])
    near = decode.rotate(x, [2], [math.pi / 4, 0.0], interleaved=True)
    assert np.allclose(near, [[[-2.0, 1.0, 3.0, 4.0]]])


@pytest.mark.parametrize("interleaved", [False, True])
def test_scores_depend_on_distance_alone(interleaved):
    rng = np.random.default_rng(0)
    w = decode.rope_frequencies(16)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    at = [float((decode.rotate(q, [p + 5], w, interleaved) * decode.rotate(k, [p], w, interleaved)).sum())
          for p in (0, 3, 1000)]
    assert np.allclose(at, at[0])


def test_scaled_frequencies():
    plain = decode.rope_frequencies(64)
    assert plain[0] == 1.0 and np.isclose(plain[-1], 10000.0 ** (-62 / 64))
    assert np.allclose(decode.rope_frequencies(64, scaling="linear", factor=4.0), plain / 4)
    base = decode.rope_frequencies(64, scaling="base", factor=4.0)
    assert base[0] == 1.0 and np.isclose(base[-1], plain[-1] / 4)
    banded = decode.rope_frequencies(64, scaling="banded", factor=8.0, original_len=8192)
    turns = 8192 * plain / (2 * math.pi)
    assert np.allclose(banded[turns >= 4], plain[turns >= 4]) and np.allclose(banded[turns <= 1], plain[turns <= 1] / 8)
    assert np.all(banded <= plain) and np.all(banded >= plain / 8)


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(interleaved):
    rng = np.random.default_rng(1)
    w = decode.rope_frequencies(8)
    x, g = rng.standard_normal((3, 2, 10)), rng.standard_normal((3, 2, 10))
    pos = [0, 7, 100]
    grad = decode.rotate(g, pos, w, interleaved, 1.25, inverse=True)
    grad[..., 8:] = g[..., 8:]
    for idx in [(0, 0, 0), (1, 1, 3), (2, 0, 7), (2, 1, 9)]:
        d = np.zeros_like(x)
        d[idx] = 1e-6
        f = [float((g * decode.rotate(x + e * d, pos, w, interleaved, 1.25)).sum()) for e in (1, -1)]
        assert np.isclose((f[0] - f[1]) / 2e-6, grad[idx], atol=1e-6)


def test_attention_by_hand():
    k = [np.array([[[0.0]], [[math.log(3.0)]], [[50.0]]])]
    v = [np.array([[[1.0]], [[5.0]], [[-100.0]]])]
    q = np.array([[[1.0]]])
    out, lse, mass, span = decode.attend(q, k, v, [2], 1, 1.0)
    assert np.isclose(out[0, 0, 0], 4.0) and np.isclose(lse[0, 0], math.log(4.0)) and np.isclose(mass[0, 0, 0], 4.0)
    out, lse, _, _ = decode.attend(q, k, v, [2], 1, 1.0, window=1)
    assert out[0, 0, 0] == 5.0 and np.isclose(lse[0, 0], math.log(3.0))
    for empty in (dict(lengths=[0]), dict(lengths=[2], starts=[2])):
        out, lse, _, _ = decode.attend(q, k, v, new_tokens=1, scale=1.0, **empty)
        assert out[0, 0, 0] == 0.0 and lse[0, 0] == -np.inf
    two = np.array([[[0.0]], [[0.0]]])       # two new tokens: the first sees one key fewer
    out, lse, _, _ = decode.attend(two, k, v, [2], 2, 1.0)
    assert out[0, 0, 0] == 1.0 and out[1, 0, 0] == 3.0 and lse[0, 0] == 0.0


def test_heads_share_keys_in_order():
    rng = np.random.default_rng(2)
    k, v = [rng.standard_normal((5, 2, 4))], [rng.standard_normal((5, 2, 4))]
    q = rng.standard_normal((1, 6, 4))
    out, _, _, _ = decode.attend(q, k, v, [5], 1, 0.5)
    for h in range(6):
        alone, _, _, _ = decode.attend(q[:, h:h + 1], [k[0][:, h // 3:h // 3 + 1]], [v[0][:, h // 3:h // 3 + 1]], [5], 1, 0.5)
        assert np.allclose(out[:, h], alone[:, 0])
