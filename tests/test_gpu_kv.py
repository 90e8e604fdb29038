"""The 4-bit cache's contents and pages against the oracle (GPU).  Codes,
parameters, tables and copied bytes are unique results and compared for
equality."""

import numpy as np
import pytest
import torch

from kv_helpers import Model, rows
from oracle import q4
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu


def _i(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _record(cache, layer, page, h, r):
    rec = q4.record_bytes(cache.head_dim, cache.group)
    at = (h * (cache.page_size // 32) + r) * rec
    return cache.data[layer, page, at:at + rec].cpu().numpy()


@pytest.mark.parametrize("H,D,G,ps", [(1, 64, 32, 32), (2, 64, 64, 64), (3, 128, 32, 64), (8, 128, 64, 128),
                                      (1, 128, 128, 1024), (2, 256, 32, 32), (1, 256, 128, 64)])
def test_append_writes_the_oracles_bytes(H, D, G, ps):
    """Three rows of ragged lengths from the middle of a record on, strided
    sources, in the second of two layers; untouched bytes stay."""
    cache = tq.KVCache.empty(2, 40, 5, 6, H, D, ps, G)
    cache.data.fill_(0xA5)
    first, new = [7, 0, 31], [70 if ps < 1024 else 300, 1, 2]
    seqs = _i(4, 0, 2)
    tq.tq_kv_extend(cache, cu_new=_i(0, *np.cumsum(first)), seqs=seqs)
    cu = [0, *np.cumsum(new).tolist()]
    starts = tq.tq_kv_extend(cache, cu_new=_i(*cu), seqs=seqs)
    assert starts.tolist() == first
    t = sum(new)
    src = [torch.from_numpy(rows((t, H + 1, D + 6), 3 + i)).cuda() for i in range(2)]
    k, v = (x[:, 1:, 1 + i:1 + i + D] for i, x in enumerate(src))
    before = cache.data.clone()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    tq.tq_kv_append(cache, 1, k, v, starts, seqs=seqs, cu_new=_i(*cu), max_new=max(new), d_err=err)
    assert int(err) == 0 and torch.equal(cache.data[0], before[0])
    kq, vq = q4.quantise(k.cpu().numpy(), G), q4.quantise(v.cpu().numpy(), G)
    table = cache.pages.cpu().numpy()
    touched = set()
    for row, s in enumerate(seqs.tolist()):
        for r in range((first[row] // 32), (first[row] + new[row] - 1) // 32 + 1):
            page = table[s, r * 32 // ps]
            touched.add(page)
            for h in range(H):
                got = _record(cache, 1, page, h, r % (ps // 32))
                old = np.frombuffer(b"\xa5" * got.size, np.uint8)
                pos = np.arange(r * 32, r * 32 + 32)
                on = (pos >= first[row]) & (pos < first[row] + new[row])
                at = cu[row] + pos[on] - first[row]
                want = _patched(old, on, [x[at, h] for x in kq], [x[at, h] for x in vq], D, G)
                np.testing.assert_array_equal(got, want, err_msg=f"slot {s} record {r} head {h}")
    rest = [p for p in range(40) if p not in touched]
    assert torch.equal(cache.data[1, rest], before[1, rest])


def _patched(old, on, kq, vq, D, G):
    """The record `old` with the tokens where `on` replaced."""
    def full(x, dtype):
        out = np.zeros((32, x.shape[-1]), dtype)
        out[on] = x
        return out

    new = q4.pack_record(full(kq[0], np.uint8), full(kq[1], np.float16), full(kq[2], np.float16),
                         full(vq[0], np.uint8), full(vq[1], np.float16), full(vq[2], np.float16), G)
    ones = full(np.full((int(on.sum()), D), 15, np.uint8), np.uint8)
    p = np.zeros((32, D // G), np.uint16)
    p[on] = 0xFFFF
    mask = q4.pack_record(ones, p.view(np.float16), p.view(np.float16), ones, p.view(np.float16),
                          p.view(np.float16), G)
    return (old & ~mask) | (new & mask)


@pytest.mark.parametrize("H,D,G,ps,lens", [(2, 64, 32, 32, [1, 0, 33, 200]), (1, 128, 64, 64, [129, 64, 65]),
                                           (3, 256, 128, 128, [300, 5])])
def test_read_gives_back_what_was_appended(H, D, G, ps, lens):
    m = Model(lens, H, D, G, ps)
    cu = [0, *np.cumsum(lens).tolist()]
    k, v = tq.tq_kv_read(m.cache, 0, _i(*[0] * len(lens)), cu[-1], cu_new=_i(*cu), max_new=max(lens))
    for got, want in ((k, m.k), (v, m.v)):
        w = np.concatenate(want)
        err = np.abs(got.cpu().numpy().astype(np.float64) - w)
        # one rounding to fp32, one to fp16
        assert (err <= np.abs(w) * (2.0 ** -11 + 2.0 ** -24) + 2.0 ** -25).all()
    # from the middle, one token a row, a row left out
    at = [max(0, n - 1) for n in lens]
    at[1] = -1
    k1, _ = tq.tq_kv_read(m.cache, 0, _i(*at), len(lens))
    for i, s in enumerate(at):
        assert torch.equal(k1[i], k[cu[i] + s] if s >= 0 else torch.zeros_like(k1[i]))


def test_append_values_that_are_not_finite():
    cache = tq.KVCache.empty(1, 2, 1, 2, 1, 64, 32, 32)
    starts = tq.tq_kv_extend(cache, cu_new=_i(0, 3))
    k = torch.ones((3, 1, 64), dtype=torch.float16, device="cuda")
    v = k.clone()
    k[1, 0, 40], v[2, 0, 3] = float("inf"), float("nan")
    tq.tq_kv_append(cache, 0, k, v, starts, cu_new=_i(0, 3), max_new=3)
    gk, gv = tq.tq_kv_read(cache, 0, starts, 3, cu_new=_i(0, 3), max_new=3)
    nan = torch.zeros((3, 1, 64), dtype=torch.bool)
    nan[1, 0, 32:] = True
    assert torch.equal(torch.isnan(gk).cpu(), nan) and bool((gk.cpu()[~nan] == 1).all())
    nan = torch.zeros((3, 1, 64), dtype=torch.bool)
    nan[2, 0, :32] = True
    assert torch.equal(torch.isnan(gv).cpu(), nan) and bool((gv.cpu()[~nan] == 1).all())


def test_append_refuses_and_counts():
    cache = tq.KVCache.empty(1, 3, 3, 3, 1, 64, 32, 64)
    tq.tq_kv_extend(cache, cu_new=_i(0, 40, 41, 41))
    before = cache.data.clone()
    k = torch.randn((8, 1, 64), device="cuda").half()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    # a slot outside, a position without a page, a row that is left out
    tq.tq_kv_append(cache, 0, k[:3], k[:3], _i(0, 64, -1), seqs=_i(7, 0, 1), d_err=err)
    assert int(err) == 2 and torch.equal(cache.data, before)
    # more tokens than max_new: the first two are written
    tq.tq_kv_append(cache, 0, k, k, _i(0, 0, 0), seqs=_i(0, 1, 2), cu_new=_i(0, 8, 8, 8), max_new=2, d_err=err)
    assert int(err) == 3
    a, _ = tq.tq_kv_read(cache, 0, _i(0), 2, seqs=_i(0), cu_new=_i(0, 2), max_new=2)
    c, s, m = q4.quantise(k[:2].cpu().numpy(), 64)
    np.testing.assert_allclose(a.cpu().numpy(), q4.values(c, s, m, 64), rtol=2.0 ** -11, atol=2.0 ** -24)


def test_append_counts_a_row_once_over_many_pages():
    """Pages missing here and there among the 40 that a row writes: the row
    counts once, what has pages is written."""
    cache = tq.KVCache.empty(1, 50, 1, 45, 1, 64, 32, 32)
    starts = tq.tq_kv_extend(cache, cu_new=_i(0, 1280))
    k = torch.from_numpy(rows((1280, 1, 64), 1)).cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    tq.tq_kv_append(cache, 0, k, k, starts, cu_new=_i(0, 1280), max_new=1280, d_err=err)
    assert int(err) == 0
    want, _ = tq.tq_kv_read(cache, 0, starts, 1280, cu_new=_i(0, 1280), max_new=1280)
    cache.data.fill_(0)
    cache.pages[0, [3, 39]] = -1
    tq.tq_kv_append(cache, 0, k, k, starts, cu_new=_i(0, 1280), max_new=1280, d_err=err)
    assert int(err) == 1
    got, _ = tq.tq_kv_read(cache, 0, starts, 1280, cu_new=_i(0, 1280), max_new=1280)
    want[96:128] = 0
    want[39 * 32:] = 0
    assert torch.equal(got, want)


class Both:
    """A cache on the GPU and its table in the oracle."""

    def __init__(self, n_pages, n_seqs, max_pages, ps=32, layers=2):
        self.c = tq.KVCache.empty(layers, n_pages, n_seqs, max_pages, 1, 64, ps, 64)
        self.c.data.copy_(torch.randint(0, 256, self.c.data.shape, dtype=torch.uint8, device="cuda"))
        self.o = q4.Pages(n_pages, n_seqs, max_pages, ps)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def same(self):
        np.testing.assert_array_equal(self.c.pages.cpu().numpy(), self.o.array())
        assert self.c.lens.tolist() == self.o.lens and self.c.refs.tolist() == self.o.refs
        assert int(self.err) == self.o.errors

    def extend(self, seqs, new):
        cu = _i(0, *np.cumsum(new).tolist())
        got = tq.tq_kv_extend(self.c, cu_new=cu, seqs=_i(*seqs), d_err=self.err)
        assert got.tolist() == self.o.extend(seqs, new)
        self.same()

    def free(self, seqs):
        tq.tq_kv_free(self.c, _i(*seqs), d_err=self.err)
        self.o.free(seqs)
        self.same()

    def moved(self, call):
        want = self.c.data.clone()
        call()
        for a, b in self.o.moves:
            want[:, b] = want[:, a]
        self.same()
        assert torch.equal(self.c.data, want)

    def fork(self, parents, children):
        self.o.fork(parents, children)
        self.moved(lambda: tq.tq_kv_fork(self.c, _i(*parents), _i(*children), d_err=self.err))

    def compact(self):
        live = self.o.compact()
        n = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        self.moved(lambda: tq.tq_kv_compact(self.c, n_live=n))
        assert int(n) == live


def test_pages_edge_cases():
    b = Both(8, 6, 3)
    b.compact()                                        # nothing in use
    b.extend([0, 3, 1], [40, 0, 64])
    b.extend([0, 9, -1, 0, 2], [24, 1, 1, 1, 1])       # fills slot 0's page; slots outside; a slot twice
    b.extend([0], [40])                                # past max_pages
    b.extend([4, 5], [96, 1])                          # slot 4 would take what is left, slot 5 gets none
    b.extend([4], [65])
    b.free([4])
    b.fork([0, 0, 2, 1, 2], [3, 4, 5, 5, 2])           # full pages only, full again, partial, child twice, itself
    b.extend([5, 2], [5, 40])                          # own partial pages grow
    b.fork([5], [0])                                   # child holds tokens
    b.free([3, 3, 0, 11])
    b.compact()
    b.free([0, 1, 2, 3, 4, 5])
    assert sum(b.o.refs) == 0


def test_extend_does_not_write_to_shared_pages():
    c = tq.KVCache.empty(1, 8, 3, 4, 1, 64, 32, 64)
    tq.tq_kv_extend(c, cu_new=_i(0, 40), seqs=_i(0))
    c.refs[int(c.pages[0, 1])] = 2                     # as if another slot named the last page
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert tq.tq_kv_extend(c, seqs=_i(0), d_err=err).tolist() == [-1] and int(err) == 1
    assert c.lens.tolist() == [40, 0, 0]


@pytest.mark.parametrize("seed", range(4))
def test_pages_over_many_calls(seed):
    r = np.random.default_rng(seed)
    n_seqs = 12
    b = Both(60, n_seqs, 9, ps=32 if seed % 2 else 64)
    for _ in range(40):
        pick = r.permutation(n_seqs)[:int(r.integers(1, n_seqs))].tolist()
        what = r.integers(0, 8)
        if what < 4:
            b.extend(pick, r.integers(0, 120, len(pick)).tolist())
        elif what < 5:
            b.free(pick)
        elif what < 7:
            b.fork(r.integers(0, n_seqs, len(pick)).tolist(), pick)
        else:
            b.compact()


def test_many_rows_and_a_large_pool():
    """1024 rows, a pool that takes many passes of the search for free pages,
    most of it in use."""
    n = 30000
    c = tq.KVCache.empty(1, n, 1024, 8, 1, 64, 32, 64)
    o = q4.Pages(n, 1024, 8, 32)
    r = np.random.default_rng(0)
    busy = r.random(n) < 0.9
    c.refs.copy_(torch.from_numpy(busy.astype(np.int32)))
    o.refs = [int(x) for x in busy]
    new = r.integers(0, 200, 1024)
    got = tq.tq_kv_extend(c, cu_new=_i(0, *np.cumsum(new).tolist()))
    want = o.extend(list(range(1024)), new.tolist())
    assert got.tolist() == want and -1 in want
    np.testing.assert_array_equal(c.pages.cpu().numpy(), o.array())
    assert c.refs.tolist() == o.refs and c.lens.tolist() == o.lens
    tq.tq_kv_free(c)
    o.free(list(range(1024)))
    assert c.refs.tolist() == o.refs and bool((c.pages == -1).all())
    data = torch.randint(0, 256, c.data.shape, dtype=torch.uint8, device="cuda")
    c.data.copy_(data)
    tq.tq_kv_compact(c)
    o.compact()
    for a, d in o.moves[:: 97]:
        assert torch.equal(c.data[0, d], data[0, a])
    assert c.refs.tolist() == o.refs


def test_copy_pages():
    c = tq.KVCache.empty(3, 9, 1, 1, 2, 128, 64, 32)
    c.data.copy_(torch.randint(0, 256, c.data.shape, dtype=torch.uint8, device="cuda"))
    want = c.data.clone()
    want[:, [0, 8]] = want[:, [5, 2]]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    tq.tq_kv_copy_pages(c, _i(5, 2, -1, 4, 3), _i(0, 8, 1, 9, 3), d_err=err)
    assert torch.equal(c.data, want) and int(err) == 2


def test_refusals():
    c = tq.KVCache.empty(1, 4, 2, 2, 1, 64, 32, 64)
    k = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda")
    for bad in (dict(k=k.float()), dict(k=k[..., ::2]), dict(v=k[:1]), dict(k=k.expand(2, 2, 64))):
        kw = dict(dict(k=k, v=k), **bad)
        with pytest.raises(ValueError):
            tq.tq_kv_append(c, 0, kw["k"], kw["v"], _i(0, 0))
    for layer in (-1, 1):
        with pytest.raises(tq.TqError) as e:
            tq.tq_kv_append(c, layer, k, k, _i(0, 0))
        assert e.value.status == 2
    with pytest.raises(tq.TqError):
        tq.tq_kv_append(c, 0, k, k, _i(0, 0, 0))       # more rows than slots
    with pytest.raises(ValueError):
        tq.tq_kv_extend(c, cu_new=_i(0, 1), seqs=_i(0, 1))
    with pytest.raises(ValueError):
        tq.KVCache(c.data[:, :, :-16].contiguous(), c.pages, c.lens, c.refs, 1, 64, 32, 64)
    for kw in (dict(page_size=48), dict(head_dim=96), dict(group=128)):
        with pytest.raises(tq.TqError):
            tq.KVCache.empty(1, 4, 2, 2, 1, **dict(dict(head_dim=64, page_size=32, group=64), **kw))
    with pytest.raises(tq.TqError) as e:
        tq.tq_kv_compact(c, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 2
