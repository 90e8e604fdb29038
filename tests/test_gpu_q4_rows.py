"""Products with 4-bit weights of one to four rows, over every number of row
tiles a workgroup takes (GPU): few outputs, more than 8192 and 32768, numbers
of tiles that the workgroups do not divide.  Tolerances as in test_gpu_q4.py."""

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2609_09240_amd import tq
from test_gpu_q4 import U, _random, _upload

pytestmark = pytest.mark.gpu

SIZES = [(100, 1152, 32), (513, 700, 64), (8192, 129, 128), (8193, 260, 64), (8225, 128, 128), (32753, 300, 32),
         (32769, 130, 64), (32785, 257, 128), (32801, 96, 32)]


def _guarded(B, n, dtype):
    """Y [B, n] with memory behind it that must stay as it is."""
    buf = torch.full((B * n + 512,), 7.0, dtype=dtype, device="cuda")
    return buf, buf[:B * n].view(B, n)


@pytest.mark.parametrize("B", [1, 2, 3, 4])
@pytest.mark.parametrize("n,k,group", SIZES)
def test_exact_sums_are_equal(n, k, group, B):
    """Whole inputs and offsets, scales that are powers of two: every partial
    sum is a whole multiple of 1/4 below 2^22, exact in fp32 in any order."""
    r = np.random.default_rng(B * 1000 + n)
    ng = -(-k // group)
    codes = r.integers(0, 16, (n, k)).astype(np.uint8)
    s = r.choice([0.25, 0.5, 1.0, -0.5], (n, ng)).astype(np.float16)
    m = r.integers(-8, 9, (n, ng)).astype(np.float16)
    x = r.integers(-3, 4, (B, k)).astype(np.float16)
    buf, y = _guarded(B, n, torch.float32)
    tq.tq_q4_gemm(_upload(codes, s, m, group), torch.from_numpy(x).cuda(), Y=y, out_f32=True)
    np.testing.assert_array_equal(y.cpu().numpy().astype(np.float64), q4.gemm(codes, s, m, group, x))
    assert bool((buf[B * n:] == 7).all())


@pytest.mark.parametrize("B", [1, 2, 3, 4])
@pytest.mark.parametrize("n,k,group", [(200, 3000, 64), (8209, 1000, 128), (32817, 500, 64)])
def test_products_within_the_bound(n, k, group, B):
    codes, s, m = _random(n, k, group, n + k)
    x = np.random.default_rng(B).standard_normal((B, k)).astype(np.float16)
    mat, xd = _upload(codes, s, m, group), torch.from_numpy(x).cuda()
    want, terms = q4.gemm(codes, s, m, group, x), q4.gemm_scale(codes, s, m, group, x)
    bound = 2 * (k + 64) * U * terms
    err = np.abs(tq.tq_q4_gemm(mat, xd, out_f32=True).cpu().numpy().astype(np.float64) - want)
    assert (err <= bound).all() and np.linalg.norm(err) <= 64 * U * np.linalg.norm(terms)
    buf, y = _guarded(B, n, torch.float16)
    tq.tq_q4_gemm(mat, xd, Y=y)
    err = np.abs(y.cpu().numpy().astype(np.float64) - want)
    assert (err <= bound * (1 + 2.0 ** -11) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25).all()
    assert bool((buf[B * n:] == 7).all())


@pytest.mark.parametrize("n", [40, 8209, 32785])
@pytest.mark.parametrize("B", [1, 2, 4])
def test_outputs_that_are_not_finite(n, B):
    """Infinite and NaN inputs and parameters, a weight of 0 under an infinity."""
    codes, s, m = _random(n, 300, 64, 9)
    codes[n - 3, 7], m[n - 3, 0] = 0, 0.0
    s[n - 1, 4] = np.nan
    x = np.random.default_rng(4).standard_normal((B, 300)).astype(np.float16)
    x[B - 1, 7] = np.inf
    got = tq.tq_q4_gemm(_upload(codes, s, m, 64), torch.from_numpy(x).cuda(), out_f32=True).cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = x.astype(np.float64) @ q4.values(codes, s, m, 64).T
    assert np.isnan(want[B - 1, n - 3]) and np.isnan(want[:, n - 1]).all()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    np.testing.assert_array_equal(got[inf], want[inf])
