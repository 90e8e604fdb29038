"""Pins of oracle/decode.py against closed forms and elementary Python (CPU)."""

import math

import numpy as np
import pytest

from oracle import decode, q4


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_is_a_complex_product(adjacent, inverse):
    r = np.random.default_rng(0)
    x = r.standard_normal((5, 3, 20))
    freq = (100.0 ** (-np.arange(8) / 8)).astype(np.float32)
    pos = r.integers(-1000, 10 ** 6, (3, 5))
    axis = np.array([0, 1, 2, 2, 1, 0, 0, 2])
    y = decode.rope(x, pos, freq, axis, adjacent, inverse, 1.25)
    assert (y[..., 16:] == x[..., 16:]).all()
    for i in range(8):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + 8)
        for t in range(5):
            w = 1.25 * np.exp(1j * (-1 if inverse else 1) * float(pos[axis[i], t]) * float(freq[i]))
            z = (x[t, :, a] + 1j * x[t, :, b]) * w
            np.testing.assert_allclose(y[t, :, a], z.real, atol=1e-12)
            np.testing.assert_allclose(y[t, :, b], z.imag, atol=1e-12)


def test_rope_quarter_turns():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    f = np.array([math.pi / 2, math.pi], np.float32)
    np.testing.assert_allclose(decode.rope(x, [1], f)[0, 0], [-3, -2, 1, -4], atol=1e-6)
    np.testing.assert_allclose(decode.rope(x, [1], f, adjacent=True)[0, 0], [-2, 1, -3, -4], atol=1e-6)
    # a pair whose axis is not there is only scaled
    np.testing.assert_allclose(decode.rope(x, [1], f, axis=[1, 0], scale=2.0)[0, 0], [2, -4, 6, -8], atol=2e-6)


def test_rope_far_positions_keep_relative_angles():
    """q . k depends on the distance alone, at any position."""
    r = np.random.default_rng(1)
    q, k = r.standard_normal((2, 1, 1, 64))
    f = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    near = (decode.rope(q, [7], f) * decode.rope(k, [2], f)).sum()
    far = (decode.rope(q, [2 ** 30 + 5], f) * decode.rope(k, [2 ** 30], f)).sum()
    assert abs(near - far) < 1e-5


def test_attention_with_sinks():
    r = np.random.default_rng(2)
    k, v, q = r.standard_normal((30, 8)), r.standard_normal((30, 8)), r.standard_normal((4, 8))
    for a, b in zip(decode.attention(q, k, v, 0.3, 5, 0), q4.attention(q, k, v, 0.3, 5)):
        np.testing.assert_array_equal(a, b)
    for a, b in zip(decode.attention(q, k, v, 0.3, 5, 27), q4.attention(q, k, v, 0.3)):
        np.testing.assert_array_equal(a, b)
    o, lse, p = decode.attention(q, k, v, 0.3, 5, 2)
    for i in range(4):
        seen = [j for j in range(30) if j <= 26 + i and (j > 21 + i or j < 2)]
        assert len(seen) == 7 and set(np.nonzero(p[i])[0]) == set(seen)
        w = [math.exp(0.3 * sum(q[i] * k[j])) for j in seen]
        np.testing.assert_allclose(lse[i], math.log(sum(w)))
        np.testing.assert_allclose(o[i], sum(a * v[j] for a, j in zip(w, seen)) / sum(w))


def test_shared_prefix_by_hand():
    table = [[5, 6, 7, -1], [5, 6, 8, -1], [5, 9, -1, -1], [5, 6, 7, 3], [-1] * 4]
    lens = [90, 96, 33, 100, 0]
    f = lambda seqs, groups: decode.shared_prefix(table, lens, 32, 10, seqs, groups)
    assert f([0, 1], [0, 2]) == [64, 64]
    assert f([0, 3], [0, 2]) == [90, 90]                    # a shared last page, partly filled
    assert f([0, 1, 2], [0, 3]) == [32, 32, 32]
    assert f([0, 1, 2, 3], [0, 2, 4]) == [64, 64, 32, 32]
    assert f([0, 4, 1, -1, 9], [0, 5]) == [64, 0, 64, 0, 0]
    assert f([0, 1, 3], [0, 1, 3]) == [0, 64, 64]           # alone
    assert f([0, 1, 3], [1, 3]) == [0, 64, 64]              # no group
    assert f([0, 0], [0, 2]) == [90, 90]
    assert decode.shared_prefix([[-1, 2], [-1, 2]], [40, 40], 32, 10, [0, 1], [0, 2]) == [0, 0]


def test_logprobs_closed_forms():
    lp, h, top, tlp = decode.logprobs(np.zeros((2, 8)), [[0, 7], [3, 8]], 3)
    np.testing.assert_allclose(lp[0], -math.log(8))
    assert np.isnan(lp[1, 1]) and top.tolist() == [[0, 1, 2]] * 2
    np.testing.assert_allclose(h, math.log(8))
    x = np.array([[0.0, math.log(3.0), -np.inf, 0.0]])
    lp, h, top, tlp = decode.logprobs(x, [1, ], 4)
    np.testing.assert_allclose(lp, [[math.log(0.6)]])
    np.testing.assert_allclose(h, -(0.6 * math.log(0.6) + 2 * 0.2 * math.log(0.2)))
    assert top.tolist() == [[1, 0, 3, 2]] and tlp[0, 3] == -np.inf
    np.testing.assert_allclose(decode.logprobs(x, [1], scale=2.0)[0], [[math.log(9 / 11)]])
    lp, h, top, tlp = decode.logprobs(np.full((1, 4), -np.inf), [2], 2)
    assert lp[0, 0] == -np.inf and h[0] == 0 and top.tolist() == [[0, 1]]
    lp, h, top, _ = decode.logprobs(np.array([[1.0, np.nan, 2.0, -np.inf]]), [0], 4)
    assert np.isnan(lp).all() and np.isnan(h).all() and top.tolist() == [[2, 0, 1, 3]]
