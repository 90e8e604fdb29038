"""Attention over values whose scales span fp16's range (GPU): groups with
outliers beside ordinary ones, tokens far below the largest probability, and
values that are tiny altogether.

Tolerance, with u = 2^-24, per head and group of channels, as a norm over the
group.  A logit is a sum of fewer than 64 roundings of both signs, each at
most u size, size = scale sum |q| (|s c| + |m|): taken as 8 u size, twice, for
it enters the sum that o is divided by as well.  The sums over tokens have
roundings of both signs too: 128 u of the terms.  A probability times its
scale is held to 22 bits (4 u) or to 2^-37 of the largest probability times
the group's largest scale, with either sign, under codes of at most 15: over L
tokens 15 sqrt(L) 2^-37 of those.
"""

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SHARE = 4


def _attend(k, v, q, G, scale, window=0):
    """k, v fp16 [L, D], q fp16 [n, SHARE, D]: the library's o and lse, and
    the oracle's values, offsets and scales."""
    L, D = k.shape
    c = tq.KVCache.empty(1, -(-L // 64), 1, -(-L // 64), 1, D, 64, G)
    cu = torch.tensor([0, L], dtype=torch.int32, device="cuda")
    starts = tq.tq_kv_extend(c, cu_new=cu)
    tq.tq_kv_append(c, 0, *(torch.from_numpy(x[:, None]).cuda() for x in (k, v)), starts, cu_new=cu, max_new=L)
    n = q.shape[0]
    o, lse = tq.tq_kv_attention(c, 0, torch.from_numpy(q).cuda(),
                                cu_q=torch.tensor([0, n], dtype=torch.int32, device="cuda"), max_q=n, scale=scale,
                                window=window, out_f32=True, want_lse=True)
    return o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


def _check(k, v, q, G, scale=None, window=0):
    D, L, n = k.shape[1], k.shape[0], q.shape[0]
    scale = D ** -0.5 if scale is None else scale
    o, lse = _attend(k, v, q, G, scale, window)
    kc, ks, km = q4.quantise(k, G)
    vc, vs, vm = q4.quantise(v, G)
    kv, vv = q4.values(kc, ks, km, G), q4.values(vc, vs, vm, G)
    at = np.arange(D) // G
    ksize = kc * ks.astype(np.float64)[:, at] + np.abs(km.astype(np.float64))[:, at]
    vsize = vc * vs.astype(np.float64)[:, at] + np.abs(vm.astype(np.float64))[:, at]
    for h in range(q.shape[1]):
        qh = q[:, h].astype(np.float64)
        want, wl, p = q4.attention(qh, kv, vv, scale, window)
        size = np.where(p > 0, (np.abs(qh) @ ksize.T) * abs(scale), 0).max(-1)
        term = p @ vsize
        for g in range(D // G):
            sl = slice(g * G, g * G + G)
            top = (p.max(-1) * np.where(p > 0, vs[:, g].astype(np.float64), 0).max(-1))
            bound = (132 * U + 16 * U * size) * np.linalg.norm(term[:, sl], axis=-1) \
                + 15 * np.sqrt(L) * 2.0 ** -37 * top * np.sqrt(G)
            err = np.linalg.norm((o[:, h] - want)[:, sl], axis=-1)
            assert (err <= bound).all(), (h, g, float((err / bound).max()), float((err / np.linalg.norm(term[:, sl], axis=-1)).max()))
        assert (np.abs(lse[:, h] - wl) <= (8 * size + 128 + 4 * np.abs(wl)) * U).all(), h


def _far(L, D, nats, sink, seed, n=1):
    """Keys and queries with one token `nats` above the rest, about."""
    r = np.random.default_rng(seed)
    u = np.where(np.arange(D) % 3 == 0, -1.0, 1.0)
    c = (nats * D ** -0.5) ** 0.5               # scale sum (c u)(c u) = nats
    q = (c * u + 0.3 * r.standard_normal((n, SHARE, D))).astype(np.float16)
    k = (0.2 * r.standard_normal((L, D))).astype(np.float16)
    k[sink] = (c * u).astype(np.float16)
    v = (r.standard_normal((L, D)) + r.standard_normal(D)).astype(np.float16)
    v[sink] = 0
    return k, v, q


@pytest.mark.parametrize("D,G,L", [(64, 32, 300), (64, 64, 4096), (128, 32, 4096), (128, 64, 32768), (128, 128, 4096),
                                   (256, 64, 2100), (256, 128, 2100), (256, 32, 300)])
@pytest.mark.parametrize("big", [31.0, 60000.0])
def test_outliers_beside_a_tail(D, G, L, big):
    """One token 13 nats above the others, whose own value is 0, and one token
    with a value scale of 4 or 8000 in one group: in the first record, in the
    middle (one wave, one part of a split), in the last ones, before and after
    the large probability."""
    for sink in (0, L - 7):
        for at, g in ((5, 0), (L // 2, D // G - 1), (L - 40, 0)):
            k, v, q = _far(L, D, 13.0, sink, D + L + at)
            v[at, g * G:(g + 1) * G] = np.where(np.arange(G) % 2, big, -big).astype(np.float16)
            _check(k, v, q, G)


@pytest.mark.parametrize("D,G", [(64, 32), (128, 64), (128, 128)])
def test_a_chunk_of_queries_with_outliers(D, G):
    """Rows of a tile that see the outlier and rows that do not."""
    L = 700
    k, v, q = _far(L, D, 13.0, 650, D, n=40)
    v[670, :G] = np.where(np.arange(G) % 2, 500.0, -500.0).astype(np.float16)
    _check(k, v, q, G)
    _check(k, v, q, G, window=25)


@pytest.mark.parametrize("D,G", [(64, 32), (128, 64), (128, 128), (256, 128)])
@pytest.mark.parametrize("size", [1e-2, 1e-4, 1e-5, 2e-6])
def test_tiny_values(D, G, size):
    """Values down to fp16's subnormal numbers, their scales with them."""
    r = np.random.default_rng(D + G)
    for L in (60, 5000):
        k, q = r.standard_normal((L, D)).astype(np.float16), r.standard_normal((1, SHARE, D)).astype(np.float16)
        _check(k, (size * r.standard_normal((L, D))).astype(np.float16), q, G)


@pytest.mark.parametrize("D,G", [(64, 32), (128, 64), (256, 128)])
def test_scales_that_grow_and_shrink(D, G):
    """Value scales over 30 powers of two along the tokens, in other orders in
    other groups."""
    L, r = 3000, np.random.default_rng(G)
    k, q = r.standard_normal((L, D)).astype(np.float16), r.standard_normal((1, SHARE, D)).astype(np.float16)
    e = np.linspace(-16, 14, L)
    v = np.empty((L, D), np.float16)
    for g in range(D // G):
        f = e if g % 2 == 0 else e[::-1]
        v[:, g * G:(g + 1) * G] = (2.0 ** f[:, None] * r.uniform(-1, 1, (L, G))).astype(np.float16)
    _check(k, v, q, G)
