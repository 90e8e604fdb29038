"""Plain CPU reference of the 4-bit operators (numpy, fp64): the quantiser,
where the layouts put each code and parameter, the product, attention over
cached tokens, and the page table as sequential Python.

The quantiser's definition is in fp32 (scale and code are rounded values), so
it is evaluated in np.float32 and its results are unique; everything that the
library may round along the way is fp64 here.
"""

import numpy as np

NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)   # element e of eight sits in this nibble of its word


def quantise(x, group):
    """fp16 x [..., n] -> codes uint8 [..., n], scale and offset fp16 [..., ceil(n/group)]."""
    x = np.asarray(x, dtype=np.float16)
    n = x.shape[-1]
    ng = -(-n // group)
    codes = np.zeros(x.shape, np.uint8)
    s = np.zeros(x.shape[:-1] + (ng,), np.float16)
    m = np.zeros_like(s)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for g in range(ng):
            w = x[..., g * group:(g + 1) * group].astype(np.float32)
            bad = ~np.isfinite(w).all(-1)
            lo, hi = w.min(-1), w.max(-1)
            sg = ((hi - lo) / np.float32(15)).astype(np.float16)
            sg[bad] = np.nan
            lo = np.where(bad, np.float32(np.nan), lo)
            sf = sg.astype(np.float32)[..., None]
            q = np.rint((w - lo[..., None]) / sf)
            q = np.where(sf > 0, np.clip(q, 0, 15), 0)
            codes[..., g * group:(g + 1) * group] = np.where(np.isnan(q), 0, q).astype(np.uint8)
            s[..., g], m[..., g] = sg, lo.astype(np.float16)
    return codes, s, m


def values(codes, s, m, group):
    """fp64 values of codes [..., n] with parameters [..., ceil(n/group)]."""
    n = codes.shape[-1]
    at = np.arange(n) // group
    return codes.astype(np.float64) * s.astype(np.float64)[..., at] + m.astype(np.float64)[..., at]


# ---- Matrices.

def _matrix_words(n, k):
    """Word and nibble of every element of an [n, k] matrix."""
    kb = -(-k // 128)
    r, i = np.arange(n)[:, None], np.arange(k)[None, :]
    word = (((r // 16) * kb + i // 128) * 64 + (i % 32 // 8) * 16 + r % 16) * 4 + i % 128 // 32
    return word, np.broadcast_to(np.array(NIBBLE)[i % 8], (n, k))


def pack_matrix(codes, s, m, group):
    """(code bytes, fp16 params) of the packed layout."""
    n, k = codes.shape
    nt, kb = -(-n // 16), -(-k // 128)
    words = np.zeros(nt * kb * 256, np.uint32)
    w, nib = _matrix_words(n, k)
    np.bitwise_or.at(words, w.ravel(), (codes.astype(np.uint32) << (4 * nib).astype(np.uint32)).ravel())
    ng = kb * (128 // group)
    params = np.zeros((nt, ng, 16, 2), np.float16)
    r, g = np.arange(n)[:, None], np.arange(s.shape[1])[None, :]
    params[r // 16, g, r % 16, 0] = s
    params[r // 16, g, r % 16, 1] = m
    return words.view(np.uint8), params.ravel()


def gemm(codes, s, m, group, x):
    """fp64 x [B, K] times the matrix's transpose."""
    return x.astype(np.float64) @ values(codes, s, m, group).T


def gemm_scale(codes, s, m, group, x):
    """sum_g |s| sum q |x| + |m| sum |x|: what rounding errors are relative to."""
    n = codes.shape[1]
    at = np.arange(n) // group
    w = codes.astype(np.float64) * np.abs(s.astype(np.float64))[:, at] + np.abs(m.astype(np.float64))[:, at]
    return np.abs(x.astype(np.float64)) @ w.T


# ---- Records of the cache: 32 tokens of one head.

def record_bytes(d, group):
    return 32 * (d + 8 * d // group)


def pack_record(kq, ks, km, vq, vs, vm, group):
    """codes [32, D] and fp16 parameters [32, D/group] of keys and values -> bytes."""
    d = kq.shape[1]
    words = np.zeros(8 * d, np.uint32)
    t, i = np.arange(32)[:, None], np.arange(d)[None, :]
    kw = ((t // 16 * 4 + i % 32 // 8) * 16 + t % 16) * (d // 32) + i // 32
    np.bitwise_or.at(words, kw.ravel(), (kq.astype(np.uint32) << (4 * np.array(NIBBLE)[i % 8]).astype(np.uint32)).ravel())
    vw = 4 * d + ((i // 64 * 4 + t % 16 // 4) * 16 + i % 16) * 4 + i % 64 // 16
    nib = np.broadcast_to(t // 16 * 4 + t % 4, (32, d))
    np.bitwise_or.at(words, vw.ravel(), (vq.astype(np.uint32) << (4 * nib).astype(np.uint32)).ravel())
    parts = [words.view(np.uint8)]
    for s, m in ((ks, km), (vs, vm)):
        parts.append(np.stack([s.T, m.T], -1).astype(np.float16).ravel().view(np.uint8))
    return np.concatenate(parts)


def attention(q, k, v, scale, window=0):
    """fp64 attention of one row and query head: q [n, D] the queries, k, v
    [L, D] the cached values; the queries are the last n tokens of the L (where
    n > L the first n - L sit before the cache and see nothing).  Returns
    o [n, D], lse [n] and the weights [n, L]."""
    n, L = q.shape[0], k.shape[0]
    o, lse, p = np.zeros((n, k.shape[1])), np.full(n, -np.inf), np.zeros((n, L))
    j = np.arange(L)
    for i in range(n):
        pos = L - n + i
        see = (j <= pos) & ((j > pos - window) if window else True)
        if not see.any():
            continue
        a = scale * (k[see].astype(np.float64) @ q[i].astype(np.float64))
        top = a.max()
        e = np.exp(a - top)
        p[i, see] = e / e.sum()
        lse[i] = top + np.log(e.sum())
        o[i] = p[i, see] @ v[see].astype(np.float64)
    return o, lse, p


# ---- The page table.

class Pages:
    """The table of a cache, one row after the other.  `moves` collects (src,
    dst) page copies of the last call, to be made in order."""

    def __init__(self, n_pages, n_seqs, max_pages, page_size):
        self.n_pages, self.max_pages, self.ps = n_pages, max_pages, page_size
        self.table = [[] for _ in range(n_seqs)]
        self.lens = [0] * n_seqs
        self.refs = [0] * n_pages
        self.errors = 0
        self.moves = []

    def _first(self, seqs):
        seen, out = set(), []
        for s in seqs:
            out.append(0 <= s < len(self.lens) and s not in seen)
            seen.add(s)
        return out

    def _free(self):
        return [p for p in range(self.n_pages) if self.refs[p] == 0]

    def extend(self, seqs, new):
        starts, free, used, taken = [], self._free(), 0, []
        for s, n, ok in zip(seqs, new, self._first(seqs)):
            need = 0
            if ok:
                ln = self.lens[s]
                ok = n >= 0 and ln + n <= self.max_pages * self.ps
                if ok and n > 0 and ln % self.ps:
                    ok = self.refs[self.table[s][ln // self.ps]] == 1
                if ok:
                    need = -(-(ln + n) // self.ps) - -(-ln // self.ps)
            at, used = used, used + need
            if ok and need and used > len(free):
                ok = False
            if not ok:
                self.errors += 1
                starts.append(-1)
                continue
            for p in free[at:at + need]:
                self.table[s].append(p)
                taken.append(p)
            starts.append(self.lens[s])
            self.lens[s] += n
        for p in taken:
            self.refs[p] = 1
        return starts

    def free(self, seqs):
        for s, ok in zip(seqs, self._first(seqs)):
            if not ok:
                self.errors += 1
                continue
            for p in self.table[s]:
                self.refs[p] -= 1
            self.table[s], self.lens[s] = [], 0

    def fork(self, parents, children):
        self.moves = []
        lens, table, free = list(self.lens), [list(t) for t in self.table], self._free()
        for p, c, first in zip(parents, children, self._first(children)):
            if not (first and 0 <= p < len(lens) and p != c and lens[c] <= 0):
                self.errors += 1
                continue
            full, part = lens[p] // self.ps, lens[p] % self.ps
            if part and not free:
                self.errors += 1
                continue
            self.table[c] = table[p][:full]
            for x in self.table[c]:
                self.refs[x] += 1
            if part:
                dst = free.pop(0)
                self.refs[dst] = 1
                self.moves.append((table[p][full], dst))
                self.table[c] = self.table[c] + [dst]
            self.lens[c] = lens[p]

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] <= 0]
        movers = [p for p in range(live, self.n_pages) if self.refs[p] > 0]
        self.moves = list(zip(movers, holes))
        to = dict(self.moves)
        for a, b in self.moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return live

    def array(self):
        a = np.full((len(self.table), self.max_pages), -1, np.int32)
        for s, t in enumerate(self.table):
            a[s, :len(t)] = t
        return a
