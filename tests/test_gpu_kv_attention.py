"""Attention over the 4-bit cache against the fp64 oracle (GPU).

Tolerance, with u = 2^-24.  A logit is fp32 sums of exact products: off by at
most d = 2 (D + 64) u scale sum |q| (|s c| + |m|).  The exponential and the
two halves of a probability add 2^-21 at most, the sums over L tokens
2 (L + 64) u, so that o is off by at most
    (2 d + 2^-20 + 4 (L + 64) u) sum_j p_j (|s c| + |m|)_j  +  15 L 2^-25 / l,
the last for second halves below fp16's smallest number (l = sum exp(s - max),
which divides them), and lse by d + 2^-21 + 2 (L + 64) u + 4 u |lse|.  Where
roundings are of both signs the error is far smaller: over a whole fp32
output its norm is held to 128 u of the norm of the terms.
"""

import numpy as np
import pytest
import torch

from kv_helpers import Model, rows
from oracle import q4
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _i(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _sizes(m, s, group):
    """|scale code| + |offset| of slot s's keys and values: at most |value| + 2 |offset|,
    and |offset| at most the largest magnitude of the group (it is its smallest value)."""
    out = []
    for x in (m.k[s], m.v[s]):
        g = np.abs(x).reshape(x.shape[0], x.shape[1], x.shape[2] // group, group).max(-1, initial=0.0)
        out.append(np.abs(x) + 2 * np.repeat(g, group, -1))
    return out


def check(m, q, nq, o, lse, seqs=None, window=0, scale=None, f32=True):
    """o, lse of queries q (numpy, rows after each other, nq[i] a row)."""
    H, D, G = m.H, m.D, m.G
    scale = D ** -0.5 if scale is None else scale
    hq = q.shape[1]
    o, lse = o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    errs, terms, at = [], [], 0
    for i, n in enumerate(nq):
        s = i if seqs is None else seqs[i]
        ks, vs = _sizes(m, s, G)
        L = m.k[s].shape[0]
        for h in range(hq):
            kv = h // (hq // H)
            qi = q[at:at + n, h]
            want, wl, p = q4.attention(qi, m.k[s][:, kv], m.v[s][:, kv], scale, window)
            got, gl = o[at:at + n, h], lse[at:at + n, h]
            size = (np.abs(qi.astype(np.float64)) @ ks[:, kv].T) * abs(scale)                  # [n, L]
            d = 2 * (D + 64) * U * np.where(p > 0, size, 0).max(-1, initial=0.0)[:, None]
            term = p @ vs[:, kv]
            top = p.max(-1, initial=0.0)[:, None]
            bound = (2 * d + 2.0 ** -20 + 4 * (L + 64) * U) * term + 15 * L * 2.0 ** -25 * top
            if not f32:
                bound = bound * (1 + 2.0 ** -11) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
            assert np.isfinite(got).all(), (i, h)
            err = np.abs(got - want)
            assert (err <= bound).all(), (i, h, float((err / np.maximum(bound, 1e-300)).max()))
            none = np.isneginf(wl)
            assert (got[none] == 0).all() and np.isneginf(gl[none]).all() and np.isfinite(gl[~none]).all()
            lb = d[:, 0] + 2.0 ** -21 + 2 * (L + 64) * U + 4 * U * np.abs(np.where(none, 0, wl))
            assert (np.abs(gl - wl)[~none] <= lb[~none]).all(), (i, h)
            errs.append(err)
            terms.append(term)
        at += n
    if f32:
        assert np.linalg.norm(np.concatenate(errs)) <= 128 * U * np.linalg.norm(np.concatenate(terms))


def run(m, q, nq, f32=True, seqs=None, **kw):
    cu = _i(0, *np.cumsum(nq).tolist())
    return tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda() if isinstance(q, np.ndarray) else q,
                              seqs=None if seqs is None else _i(*seqs), cu_q=cu, max_q=max(max(nq), 1), out_f32=f32,
                              want_lse=True, **kw)


@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64),
                                 (256, 128)])
@pytest.mark.parametrize("share", [1, 4, 7, 16])
def test_decode(D, G, share):
    """One token a row over every ragged end, no token at all among them."""
    lens = [1, 0, 31, 32, 33, 64, 65, 127, 200]
    m = Model(lens, 2, D, G, 32, seed=D + G)
    q = rows((len(lens), 2 * share, D), 5)
    o, lse = tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda(), out_f32=True, want_lse=True)
    check(m, q, [1] * len(lens), o, lse)
    h = tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda())
    check(m, q, [1] * len(lens), h, lse, f32=False)


@pytest.mark.parametrize("D,G,H,share,ps", [(64, 32, 1, 14, 64), (128, 64, 2, 4, 128), (256, 64, 1, 3, 32),
                                            (128, 128, 1, 1, 1024), (64, 64, 2, 40, 32)])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_many_queries(D, G, H, share, ps, window):
    """Ragged numbers of queries, none and more than there are tokens among
    them, rows of the call in another order than the slots."""
    lens = [90, 70, 5, 0, 130]
    nq = [13, 70, 9, 3, 0, 1]
    seqs = [4, 1, 2, 3, 0, 0]
    m = Model(lens, H, D, G, ps, seed=D + window)
    q = rows((sum(nq), H * share, D), 6)
    o, lse = run(m, q, nq, seqs=seqs, window=window)
    check(m, q, nq, o, lse, seqs=seqs, window=window)


@pytest.mark.parametrize("D,G,lens,nq,share,window", [
    (128, 64, [5000, 77, 1024], [1, 1, 1], 4, 0),      # a long row in many parts beside a short one
    (128, 128, [9000], [1], 8, 0),
    (64, 32, [4000], [1], 1, 700),                      # a window that starts inside a part
    (128, 32, [3000, 2999], [9, 2], 4, 0),              # several tiles, several parts
    (64, 64, [2500], [100], 2, 1000),
    (256, 128, [2100], [3], 7, 0),
])
def test_long(D, G, lens, nq, share, window):
    m = Model(lens, 2, D, G, 64, seed=7)
    q = rows((sum(nq), 2 * share, D), 8)
    o, lse = run(m, q, nq, window=window)
    check(m, q, nq, o, lse, window=window)
    for hint in (max(lens), 50, 1):                     # a hint that is too small is slower, not wrong
        o2, lse2 = run(m, q, nq, window=window, max_len=hint)
        check(m, q, nq, o2, lse2, window=window)
    assert all(torch.equal(a, b) for a, b in zip(run(m, q, nq, window=window), (o, lse)))


def test_peaked_and_far_logits():
    """Softmaxes from nearly uniform to one-hot, logits of hundreds, maxima
    that come late: the running maximum is rescaled often."""
    L = 700
    m = Model([L], 1, 64, 32, 64, seed=3)
    q = rows((8, 4, 64), 9)
    q[0] *= 0.01
    q[1] *= 40
    q[2] = 0
    for scale in (None, 0.01, -0.5, 2.0):
        o, lse = run(m, q, [8], scale=scale)
        check(m, q, [8], o, lse, scale=scale)


def test_strided_queries():
    m = Model([100, 40], 2, 128, 64, 64)
    buf = torch.full((9, 11, 140), float("nan"), dtype=torch.float16, device="cuda")
    view = buf[::2, 1:9, 3:131]
    q = rows((5, 8, 128), 4)
    view.copy_(torch.from_numpy(q))
    o, lse = run(m, view, [3, 2])
    check(m, q, [3, 2], o, lse)
    assert torch.equal(run(m, q, [3, 2])[0], o)


def test_what_may_not_be_seen_does_not_show():
    """NaN and infinite keys and values behind a query, outside its window and
    in other slots change nothing; NaN queries change their own rows only."""
    m = Model([50, 60], 1, 64, 32, 32)
    q = rows((20, 4, 64), 1)
    o, lse = run(m, q, [10, 10], window=30)
    bad = torch.full((1, 1, 64), float("nan"), dtype=torch.float16, device="cuda")
    inf = torch.full((1, 1, 64), float("inf"), dtype=torch.float16, device="cuda")
    # slot 0: query t sits at 40 + t and sees 11 + t .. 40 + t
    tq.tq_kv_append(m.cache, 0, bad, inf, _i(49), seqs=_i(0))
    tq.tq_kv_append(m.cache, 0, inf, bad, _i(11), seqs=_i(0))
    o2, lse2 = run(m, q, [10, 10], window=30)
    fine = [t for t in range(20) if t not in (0, 9)]
    assert torch.equal(o2[fine], o[fine]) and torch.equal(lse2[fine], lse[fine])
    assert bool(torch.isnan(o2[[0, 9]]).any())
    q2 = q.copy()
    q2[12, 1] = np.nan
    q2[13, 2, 5] = np.inf
    o3, lse3 = run(m, q2, [10, 10], window=30)
    same = torch.ones((20, 4), dtype=torch.bool, device="cuda")
    same[12, 1] = same[13, 2] = False
    assert torch.equal(o3[10:][same[10:]], o2[10:][same[10:]]) and bool(torch.isnan(o3[12, 1]).all())


def test_positions_without_a_page_are_left_out():
    m = Model([96], 1, 64, 64, 32)
    q = rows((1, 2, 64), 2)
    m.cache.pages[0, 1] = -1
    o, lse = run(m, q, [1])
    m.cache.pages[0, 1] = 10 ** 6
    assert torch.equal(run(m, q, [1])[0], o)
    keep = np.r_[0:32, 64:96]
    m.k[0], m.v[0] = m.k[0][keep], m.v[0][keep]
    check(m, q, [1], o, lse)


def test_slots_outside_and_bad_offsets_read_nothing():
    m = Model([40, 40], 1, 64, 64, 32)
    q = torch.from_numpy(rows((3, 1, 64), 2)).cuda()
    o, lse = tq.tq_kv_attention(m.cache, 0, q, seqs=_i(5, -1, 1), want_lse=True)
    assert bool((o[:2] == 0).all()) and bool(torch.isneginf(lse[:2]).all())
    check(m, q.cpu().numpy()[2:], [1], o[2:], lse[2:], seqs=[1], f32=False)
    o = torch.full((3, 1, 64), 9.0, dtype=torch.float16, device="cuda")
    tq.tq_kv_attention(m.cache, 0, q, cu_q=_i(-5, 2, 900), max_q=4, o=o)
    assert bool((o[:2] == 9).all()) and bool((o[2] != 9).any())


def test_layers_and_offsets_past_32_bits():
    """Pages whose bytes lie beyond 4 GiB of the pool, in the second layer."""
    pb = int(q4.record_bytes(128, 128)) * 8 * 32
    n = (5 << 30) // pb
    c = tq.KVCache.empty(2, n, 1, 4, 8, 128, 1024, 128)
    c.refs[:n - 3] = 1
    starts = tq.tq_kv_extend(c, cu_new=_i(0, 2050))
    assert c.pages.tolist() == [[n - 3, n - 2, n - 1, -1]]
    k, v = (rows((2050, 8, 128), 30 + i) for i in range(2))
    tq.tq_kv_append(c, 1, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), starts, cu_new=_i(0, 2050),
                    max_new=2050)
    m = Model.__new__(Model)
    m.H, m.D, m.G, m.cache = 8, 128, 128, c
    m.k, m.v = ([q4.values(*q4.quantise(x, 128), 128)] for x in (k, v))
    q = rows((1, 32, 128), 3)
    o, lse = tq.tq_kv_attention(c, 1, torch.from_numpy(q).cuda(), out_f32=True, want_lse=True)
    check(m, q, [1], o, lse)


def test_streams_and_graphs():
    m = Model([700, 3, 0], 2, 128, 64, 64)
    q = torch.randn((3, 8, 128), dtype=torch.float16, device="cuda")
    want = tq.tq_kv_attention(m.cache, 0, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tq.tq_kv_attention(m.cache, 0, q, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    # A decode step of the cache: room for one token, its key and value, attention.
    new = [torch.randn((3, 2, 128), dtype=torch.float16, device="cuda") for _ in range(2)]
    o = torch.empty_like(want)
    starts = torch.empty(3, dtype=torch.int32, device="cuda")

    def step():
        tq.tq_kv_extend(m.cache, starts=starts)
        tq.tq_kv_append(m.cache, 0, *new, starts)
        tq.tq_kv_attention(m.cache, 0, q, o=o, max_len=800)

    saved = [t.clone() for t in m.cache._buffers()]
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()

    def restore():
        for t, s in zip(m.cache._buffers(), saved):
            t.copy_(s)

    eager = []
    restore()
    for i in range(4):
        for x in new:
            x.copy_(torch.full_like(x, 0.25 * i) + torch.arange(128, device="cuda") / 64)
        step()
        torch.cuda.synchronize()
        eager.append((o.clone(), m.cache.lens.clone()))
    restore()
    for i in range(4):
        for x in new:
            x.copy_(torch.full_like(x, 0.25 * i) + torch.arange(128, device="cuda") / 64)
        o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager[i][0]) and torch.equal(m.cache.lens, eager[i][1]), i


def test_refusals():
    m = Model([2000], 2, 128, 64, 64)
    q = torch.zeros((1, 8, 128), dtype=torch.float16, device="cuda")
    for bad in (q.float(), q[..., :64], q[:, :, ::2], q.cpu()):
        with pytest.raises(ValueError):
            tq.tq_kv_attention(m.cache, 0, bad)
    for kw, status in ((dict(layer=1), 2), (dict(q=q[:, :3]), 2), (dict(window=-1), 2), (dict(max_len=-1), 2),
                       (dict(max_q=0, cu_q=_i(0, 1)), 2), (dict(scale=float("inf")), 2)):
        with pytest.raises(tq.TqError) as e:
            tq.tq_kv_attention(m.cache, **dict(dict(layer=0, q=q), **kw))
        assert e.value.status == status, kw
    with pytest.raises(tq.TqError) as e:
        tq.tq_kv_attention(m.cache, 0, q, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 2
    with pytest.raises(ValueError):
        tq.tq_kv_attention(m.cache, 0, q.expand(2, 8, 128), seqs=_i(0))
