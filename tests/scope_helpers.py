"""Shared helpers of the tests of attention with sinks and over shared
prefixes: the check against the fp64 oracle, and a cache with branches.

Tolerance: that of tests/test_gpu_kv_attention.py, with u = 2^-24 and
d = 2 (D + 64) u scale sum |q| (|s c| + |m|):
    (2 d + 2^-20 + 4 (L + 64) u) sum_j p_j (|s c| + |m|)_j + 15 L 2^-25 / l,
and 8 u for each part of the shared tokens' sums that is taken up (two weights, two
products and a sum, of u or 2 u each), of which there are 32 at most: 256 u.
"""

import numpy as np
import torch

from kv_helpers import Model
from oracle import decode
from paper_2609_09240_amd import tq

U = 2.0 ** -24


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def sizes(m, s, group):
    """|scale code| + |offset| of slot s's keys and values: at most |value| + 2 |offset|,
    and |offset| at most the largest magnitude of the group (it is its smallest value)."""
    out = []
    for x in (m.k[s], m.v[s]):
        g = np.abs(x).reshape(x.shape[0], x.shape[1], x.shape[2] // group, group).max(-1, initial=0.0)
        out.append(np.abs(x) + 2 * np.repeat(g, group, -1))
    return out


def check(m, q, nq, o, lse, seqs=None, window=0, sinks=0, scale=None, f32=True, max_q=None):
    """o, lse of queries q (numpy, rows after each other, nq[i] a row).  Slots
    outside the cache hold nothing; tokens past max_q are not looked at."""
    H, D, G = m.H, m.D, m.G
    scale = D ** -0.5 if scale is None else scale
    hq = q.shape[1]
    o, lse = o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    at = 0
    for i, n in enumerate(nq):
        s = i if seqs is None else seqs[i]
        there = 0 <= s < len(m.k)
        ks, vs = sizes(m, s, G) if there else (np.zeros((0, H, D)),) * 2
        mk, mv = (m.k[s], m.v[s]) if there else (np.zeros((0, H, D)),) * 2
        L = mk.shape[0]
        keep = n if max_q is None else min(n, max_q)
        for h in range(hq):
            kv = h // (hq // H)
            qi = q[at:at + n, h]
            want, wl, p = (x[:keep] for x in decode.attention(qi, mk[:, kv], mv[:, kv], scale, window, sinks))
            got, gl = o[at:at + keep, h], lse[at:at + keep, h]
            size = (np.abs(qi[:keep].astype(np.float64)) @ ks[:, kv].T) * abs(scale)               # [keep, L]
            d = 2 * (D + 64) * U * np.where(p > 0, size, 0).max(-1, initial=0.0)[:, None]
            term = p @ vs[:, kv]
            top = p.max(-1, initial=0.0)[:, None]
            bound = (2 * d + 2.0 ** -20 + (256 + 4 * (L + 64)) * U) * term + 15 * L * 2.0 ** -25 * top
            if not f32:
                bound = bound * (1 + 2.0 ** -11) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
            assert np.isfinite(got).all(), (i, h)
            err = np.abs(got - want)
            assert (err <= bound).all(), (i, h, float((err / np.maximum(bound, 1e-300)).max()))
            none = np.isneginf(wl)
            assert (got[none] == 0).all() and np.isneginf(gl[none]).all() and np.isfinite(gl[~none]).all()
            lb = d[:, 0] + 2.0 ** -21 + (256 + 2 * (L + 64)) * U + 4 * U * np.abs(np.where(none, 0, wl))
            assert (np.abs(gl[~none] - wl[~none]) <= lb[~none]).all(), (i, h)
        at += n


class Branches(Model):
    """Slots 0 .. P-1 hold prompts of the given lengths; slot P + i is forked
    from slot parents[i] and gets tails[i] tokens of its own."""

    def __init__(self, prompts, parents, tails, H, D, G, ps, seed=0, n_layers=1):
        self.H, self.D, self.G, self.ps = H, D, G, ps
        held = list(prompts) + [prompts[p] + t for p, t in zip(parents, tails)]
        need = [-(-n // ps) for n in held]
        self.cache = tq.KVCache.empty(n_layers, sum(need) + 2, len(held), max(need + [1]) + 1, H, D, ps, G)
        self.cache.data.fill_(0xFF)
        self.k, self.v = [], []
        P = len(prompts)
        self.append(list(prompts) + [0] * len(parents), 0, seed)
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        if parents:
            tq.tq_kv_fork(self.cache, i32(*parents), i32(*range(P, len(held))), d_err=err)
        for i, p in enumerate(parents):
            self.k[P + i], self.v[P + i] = self.k[p].copy(), self.v[p].copy()
        self.append([0] * P + list(tails), 0, seed + 1)
        assert int(err) == 0 and self.cache.lens.tolist() == held
        self.kids = list(range(P, len(held)))
