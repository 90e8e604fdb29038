"""Attention over the 4-bit cache with a window and sinks, against the fp64
oracle (GPU; tolerance: scope_helpers.py)."""

import numpy as np
import pytest
import torch

from kv_helpers import Model, rows
from paper_2609_09240_amd import tq
from scope_helpers import check, i32

pytestmark = pytest.mark.gpu


def run(m, q, nq, f32=True, seqs=None, **kw):
    cu = i32(0, *np.cumsum(nq).tolist())
    return tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda() if isinstance(q, np.ndarray) else q,
                              seqs=None if seqs is None else i32(*seqs), cu_q=cu, max_q=max(max(nq), 1), out_f32=f32,
                              want_lse=True, **kw)


@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64),
                                 (256, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (40, 4), (33, 64), (100, 37), (1000, 5), (32, 1000)])
def test_decode(D, G, window, sinks):
    """One token a row over every ragged end, no token at all among them; sinks
    and windows that meet, that do not, and that are longer than the rows."""
    lens = [1, 0, 31, 32, 33, 64, 65, 100, 127, 133, 200, 333]
    m = Model(lens, 2, D, G, 32, seed=D + G)
    q = rows((len(lens), 8, D), 5)
    kw = dict(window=window, sinks=sinks)
    o, lse = tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda(), out_f32=True, want_lse=True, **kw)
    check(m, q, [1] * len(lens), o, lse, **kw)
    h = tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda(), **kw)
    check(m, q, [1] * len(lens), h, lse, f32=False, **kw)


@pytest.mark.parametrize("D,G,H,share,ps", [(64, 32, 1, 14, 64), (128, 64, 2, 4, 128), (256, 64, 1, 3, 32),
                                            (128, 128, 1, 1, 1024), (64, 64, 2, 40, 32)])
@pytest.mark.parametrize("window,sinks", [(1, 3), (20, 33), (70, 1)])
def test_many_queries(D, G, H, share, ps, window, sinks):
    """Ragged numbers of queries, none and more than there are tokens among
    them, rows of the call in another order than the slots."""
    lens = [190, 70, 5, 0, 230]
    nq = [13, 70, 9, 3, 0, 1, 60]
    seqs = [4, 1, 2, 3, 0, 0, 4]
    m = Model(lens, H, D, G, ps, seed=D + window)
    q = rows((sum(nq), H * share, D), 6)
    o, lse = run(m, q, nq, seqs=seqs, window=window, sinks=sinks)
    check(m, q, nq, o, lse, seqs=seqs, window=window, sinks=sinks)


@pytest.mark.parametrize("D,G,lens,nq,share,window,sinks", [
    (128, 64, [5000, 77, 1024], [1, 1, 1], 4, 2000, 4),     # a long row in many parts beside a short one
    (128, 128, [9000], [1], 8, 3000, 700),                  # parts that hold sinks and window
    (64, 32, [4000], [1], 1, 700, 1),
    (128, 32, [3000, 2999], [9, 2], 4, 1500, 100),          # several tiles, several parts
    (64, 64, [2500], [100], 2, 1000, 65),
    (256, 128, [2100], [3], 7, 900, 900),
])
def test_long(D, G, lens, nq, share, window, sinks):
    m = Model(lens, 2, D, G, 64, seed=7)
    q = rows((sum(nq), 2 * share, D), 8)
    kw = dict(window=window, sinks=sinks)
    o, lse = run(m, q, nq, **kw)
    check(m, q, nq, o, lse, **kw)
    for hint in (max(lens), 50, 1):                         # a hint that is too small is slower, not wrong
        o2, lse2 = run(m, q, nq, max_len=hint, **kw)
        check(m, q, nq, o2, lse2, **kw)
    assert all(torch.equal(a, b) for a, b in zip(run(m, q, nq, **kw), (o, lse)))


def test_sinks_that_change_nothing():
    """Without a window, and where the window reaches the sinks."""
    m = Model([300, 5], 2, 128, 64, 64)
    q = rows((2, 8, 128), 1)
    a, b = run(m, q, [1, 1], sinks=9), run(m, q, [1, 1])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    o, lse = run(m, q, [1, 1], sinks=9, window=1000)         # (sums in another order)
    check(m, q, [1, 1], o, lse)


@pytest.mark.parametrize("sinks", [2 ** 31 - 1, 2 ** 31 - 30, 2 ** 31 - 31, 2 ** 31 - 32, 2 ** 31 - 33])
@pytest.mark.parametrize("nq", [[1, 1, 1], [3, 40, 1]])
def test_as_many_sinks_as_there_are_numbers(sinks, nq):
    """Every token, then: as if there were no window, in one part and in several."""
    m = Model([5000, 70, 1], 2, 128, 64, 64, seed=3)
    q = rows((sum(nq), 8, 128), 6)
    for window in (1, 40, 2 ** 31 - 1):
        for hint in (0, 100):
            o, lse = run(m, q, nq, window=window, sinks=sinks, max_len=hint)
            check(m, q, nq, o, lse)


def test_what_may_not_be_seen_does_not_show():
    """NaN and infinite keys and values between the sinks and the window."""
    m = Model([200], 1, 64, 32, 32)
    q = rows((3, 4, 64), 1)
    kw = dict(window=50, sinks=35)
    o, lse = run(m, q, [3], **kw)
    bad = torch.full((1, 1, 64), float("nan"), dtype=torch.float16, device="cuda")
    inf = torch.full((1, 1, 64), float("inf"), dtype=torch.float16, device="cuda")
    # queries at 197, 198, 199 see 0 .. 34 and 148 .. 197, 149 .. 198, 150 .. 199
    for at, k, v in ((35, bad, inf), (63, inf, bad), (100, bad, bad), (147, bad, inf), (199, inf, inf), (148, bad, bad)):
        tq.tq_kv_append(m.cache, 0, k, v, i32(at), seqs=i32(0))
    o2, lse2 = run(m, q, [3], **kw)
    assert torch.equal(o2[1], o[1]) and torch.equal(lse2[1], lse[1])
    assert bool(torch.isnan(o2[0]).any()) and bool(torch.isnan(o2[2]).any())


def test_pages_that_are_gone_between_sinks_and_window():
    """A stream whose middle pages were given back: the table names none."""
    m = Model([500], 1, 128, 64, 32)
    q = rows((1, 4, 128), 2)
    kw = dict(window=100, sinks=4)
    o, lse = run(m, q, [1], **kw)
    m.cache.pages[0, 1:12] = -1
    assert all(torch.equal(a, b) for a, b in zip(run(m, q, [1], **kw), (o, lse)))
    check(m, q, [1], o, lse, **kw)


def test_workspaces_streams_and_graphs():
    m = Model([5000, 3, 0], 2, 128, 64, 64)
    q = torch.randn((3, 8, 128), dtype=torch.float16, device="cuda")
    kw = dict(window=3000, sinks=100, max_len=5000)
    need = tq.tq_kv_attention_workspace_bytes(m.cache, 3, 8, max_len=5000, window=3000, sinks=100)
    assert need > 0
    want = tq.tq_kv_attention(m.cache, 0, q, **kw)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:tq.WORKSPACE_COUNT_BYTES] = 0
    for _ in range(2):
        assert torch.equal(tq.tq_kv_attention(m.cache, 0, q, workspace=ws, **kw), want)
    with pytest.raises(tq.TqError):
        tq.tq_kv_attention(m.cache, 0, q, workspace=ws[:need - 16].clone(), **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tq.tq_kv_attention(m.cache, 0, q, stream=side, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    o = torch.empty_like(want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tq.tq_kv_attention(m.cache, 0, q, o=o, **kw)
    for i in range(3):
        q.copy_(torch.randn_like(q))
        want = tq.tq_kv_attention(m.cache, 0, q, **kw)
        o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), i


def test_refusals():
    m = Model([100], 1, 64, 64, 32)
    q = torch.zeros((1, 2, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(tq.TqError) as e:
        tq.tq_kv_attention(m.cache, 0, q, window=5, sinks=-1)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        tq.tq_kv_attention(m.cache, 0, q, window=5, sinks=1 << 33)
    with pytest.raises(tq.TqError) as e:
        tq.tq_kv_attention(m.cache, 1, q, window=5, sinks=1)
    assert e.value.status == 2
