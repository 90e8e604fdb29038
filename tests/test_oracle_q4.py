"""The 4-bit oracle against brute force and closed forms (CPU only)."""

from fractions import Fraction

import numpy as np
import pytest

from oracle import q4


def test_quantiser_on_values_it_holds_exactly():
    """Sixteen equally spaced values come back as they were."""
    for step in (0.25, 1.0, 8.0):
        x = (np.arange(32) % 16 * step - 2.0).astype(np.float16)[None]
        c, s, m = q4.quantise(x, 32)
        assert s[0, 0] == step and m[0, 0] == -2.0
        np.testing.assert_array_equal(c[0], np.arange(32) % 16)
        np.testing.assert_array_equal(q4.values(c, s, m, 32)[0], x[0].astype(np.float64))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantiser_error_and_short_groups(group):
    """Every value is within half a step, and what rounding the scale to fp16
    adds over 15 steps, of what it was."""
    r = np.random.default_rng(group)
    x = (r.standard_normal((5, 300)) * 3).astype(np.float16)
    c, s, m = q4.quantise(x, group)
    assert s.shape == (5, -(-300 // group)) and c.max() == 15 and c.min() == 0
    at = np.arange(300) // group
    sf = s.astype(np.float64)[:, at]
    assert (np.abs(q4.values(c, s, m, group) - x.astype(np.float64)) <= sf * (0.5 + 15 * 2.0 ** -11) + 1e-7).all()


def test_quantiser_special_groups():
    x = np.zeros((5, 32), np.float16)
    x[1] = 7.5
    x[2, 3] = np.inf
    x[3, 4] = np.nan
    x[4, 0], x[4, 1] = 65504, -65504
    c, s, m = q4.quantise(x, 32)
    assert (c[:4] == 0).all()
    assert s[0, 0] == 0 and m[0, 0] == 0 and s[1, 0] == 0 and m[1, 0] == 7.5
    assert np.isnan(s[2:4]).all() and np.isnan(m[2:4]).all()
    assert np.isfinite(s[4, 0]) and c[4, 0] == 15 and c[4, 1] == 0


def test_layouts_put_every_code_in_a_place_of_its_own():
    for n, k in ((1, 1), (16, 128), (17, 129), (40, 300)):
        w, nib = q4._matrix_words(n, k)
        assert len(set((w * 8 + nib).ravel().tolist())) == n * k
        assert w.max() < -(-n // 16) * -(-k // 128) * 256
    r = np.random.default_rng(0)
    for d in (64, 128, 256):
        g = 64
        one = [r.integers(0, 16, (32, d)).astype(np.uint8) for _ in range(2)]
        p = [r.standard_normal((32, d // g)).astype(np.float16) for _ in range(4)]
        b = q4.pack_record(one[0], p[0], p[1], one[1], p[2], p[3], g)
        assert b.nbytes == q4.record_bytes(d, g)
        # every nibble of every code is there: the histogram of the bytes' nibbles is that of the codes
        nib = np.concatenate([b[:32 * d] & 15, b[:32 * d] >> 4])
        want = np.bincount(np.concatenate([one[0].ravel(), one[1].ravel()]), minlength=16)
        np.testing.assert_array_equal(np.bincount(nib, minlength=16), want)


def test_product_in_rationals():
    r = np.random.default_rng(1)
    codes = r.integers(0, 16, (3, 40)).astype(np.uint8)
    s, m = (r.standard_normal((3, 2)).astype(np.float16) for _ in range(2))
    x = r.standard_normal((2, 40)).astype(np.float16)
    y = q4.gemm(codes, s, m, 32, x)
    for b in range(2):
        for n in range(3):
            t = sum((Fraction(float(m[n, k // 32])) + Fraction(float(s[n, k // 32])) * int(codes[n, k]))
                    * Fraction(float(x[b, k])) for k in range(40))
            assert abs(y[b, n] - float(t)) <= 1e-13 * q4.gemm_scale(codes, s, m, 32, x)[b, n]


def test_attention_closed_forms():
    k = np.zeros((7, 4))
    v = np.arange(28.0).reshape(7, 4)
    o, lse, _ = q4.attention(np.ones((3, 4)), k, v, 0.5)
    np.testing.assert_allclose(o, [v[:5].mean(0), v[:6].mean(0), v.mean(0)])
    np.testing.assert_allclose(lse, np.log([5, 6, 7]))
    o, lse, _ = q4.attention(np.ones((3, 4)), k, v, 0.5, window=2)
    np.testing.assert_allclose(o, [v[3:5].mean(0), v[4:6].mean(0), v[5:7].mean(0)])
    o, lse, _ = q4.attention(np.ones((3, 4)), k[:1], v[:1], 0.5)
    assert (o[:2] == 0).all() and np.isneginf(lse[:2]).all() and (o[2] == v[0]).all()


def test_page_table():
    p = q4.Pages(6, 4, 3, 32)
    assert p.extend([0, 1, 0], [40, 32, 1]) == [0, 0, -1]      # slot 0 named twice
    assert p.table[0] == [0, 1] and p.table[1] == [2] and p.errors == 1
    p.fork([0, 0], [2, 3])
    assert p.table[2] == [0, 3] and p.table[3] == [0, 4] and p.refs == [3, 1, 1, 1, 1, 0] and p.moves == [(1, 3), (1, 4)]
    assert p.extend([2, 1, 3], [60, 1, 1]) == [-1, 32, 40]     # slot 2 would need four pages, slot 1 gets page 5
    assert p.extend([0], [30]) == [-1]                         # no page left
    p.free([0, 2])
    assert p.refs == [1, 0, 1, 0, 1, 1] and p.compact() == 4
    assert p.moves == [(4, 1), (5, 3)] and p.table == [[], [2, 3], [], [0, 1]]
