"""Activations and queries that are subnormal fp16 numbers (GPU): their products
with codes are exact like any others, so the tolerances are those of
test_gpu_q4.py and test_gpu_kv_scales.py as they stand."""

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2609_09240_amd import tq
from test_gpu_kv_scales import SHARE, _check
from test_gpu_q4 import U, _random, _upload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [1, 4, 7, 24, 64])
@pytest.mark.parametrize("e", [-14, -17, -20, -23])
def test_products(B, e):
    n, k, group = 300, 4096, 64
    codes, s, m = _random(n, k, group, 3)
    x = (np.random.default_rng(B).standard_normal((B, k)) * 2.0 ** e).astype(np.float16)
    x[-1, ::5] = (x[-1, ::5].astype(np.float32) * 2.0 ** 14).astype(np.float16)    # beside ordinary ones
    got = tq.tq_q4_gemm(_upload(codes, s, m, group), torch.from_numpy(x).cuda(), out_f32=True)
    want, terms = q4.gemm(codes, s, m, group, x), q4.gemm_scale(codes, s, m, group, x)
    err = np.abs(got.cpu().numpy().astype(np.float64) - want)
    assert (err <= 2 * (k + 64) * U * terms).all()
    for b in range(B):
        assert np.linalg.norm(err[b]) <= 64 * U * np.linalg.norm(terms[b]), b


@pytest.mark.parametrize("D,G", [(64, 32), (128, 64), (256, 128)])
@pytest.mark.parametrize("e", [-15, -20])
def test_queries(D, G, e):
    """The scale makes up for them, so that the logits are ordinary."""
    r = np.random.default_rng(D)
    for L in (50, 3000):
        k, v = (r.standard_normal((L, D)).astype(np.float16) for _ in range(2))
        q = (r.standard_normal((3, SHARE, D)) * 2.0 ** e).astype(np.float16)
        _check(k, v, q, G, scale=2.0 ** -e * D ** -0.5)
