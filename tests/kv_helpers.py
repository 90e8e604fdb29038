"""Shared helpers of the 4-bit cache tests: a cache on the GPU with its page
table and fp16 contents on the CPU."""

import numpy as np
import torch

from oracle import q4
from paper_2609_09240_amd import tq


def rows(shape, seed):
    x = np.random.default_rng(seed).standard_normal(shape).astype(np.float16)
    x[..., 3::37] *= 4.0
    return x


class Model:
    """Slots filled with the given lengths through tq_kv_extend and
    tq_kv_append, and the values that the oracle's quantiser gives for them
    (fp64, layer 0): k[s], v[s] of shape [len, H, D]."""

    def __init__(self, lens, H, D, G, ps, n_layers=1, spare=3, seed=0, layer=0, poison=True):
        self.H, self.D, self.G, self.ps = H, D, G, ps
        need = [-(-n // ps) for n in lens]
        self.cache = tq.KVCache.empty(n_layers, sum(need) + spare, len(lens), max(need + [1]) + 1, H, D, ps, G)
        # what was never written reads as NaN parameters and codes of 15
        self.cache.data.fill_(0xFF if poison else 0)
        self.k, self.v = [], []
        # in two goes, so that records are filled in parts and pages of the slots alternate
        for part in (0, 1):
            new = [n // 3 if part == 0 else n - n // 3 for n in lens]
            self.append(new, layer, seed + part)

    def append(self, new, layer=0, seed=0):
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        t = int(cu[-1])
        cud = torch.from_numpy(cu).cuda()
        starts = tq.tq_kv_extend(self.cache, cu_new=cud)
        if t:
            k, v = rows((t, self.H, self.D), 2 * seed + 11), rows((t, self.H, self.D), 2 * seed + 12)
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            tq.tq_kv_append(self.cache, layer, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), starts,
                            cu_new=cud, max_new=max(new), d_err=err)
            assert int(err) == 0
        for s in range(len(new)):
            if len(self.k) <= s:
                self.k.append(np.zeros((0, self.H, self.D)))
                self.v.append(np.zeros((0, self.H, self.D)))
            if new[s]:
                for mine, x in ((self.k, k), (self.v, v)):
                    c, sc, m = q4.quantise(x[cu[s]:cu[s + 1]], self.G)
                    mine[s] = np.concatenate([mine[s], q4.values(c, sc, m, self.G)])
        return starts
