"""Attention of rows that share the pages of a prefix, and the prefix that they
share, against the fp64 oracle (GPU; tolerance: scope_helpers.py)."""

import numpy as np
import pytest
import torch

from kv_helpers import rows
from oracle import decode
from paper_2609_09240_amd import tq
from scope_helpers import Branches, check, i32

pytestmark = pytest.mark.gpu

FEW, MANY = dict(max_prefix=2000), dict(max_prefix=1 << 20)   # short caches attended together all the same, in few or many parts


def run(m, q, nq, seqs, groups=None, prefix=None, f32=True, **kw):
    seqs_t = i32(*seqs)
    g = None if groups is None else i32(*groups)
    if prefix is None:
        prefix = tq.tq_kv_shared_prefix(m.cache, groups=g, seqs=seqs_t)
        want = decode.shared_prefix(m.cache.pages.tolist(), m.cache.lens.tolist(), m.ps, m.cache.refs.numel(), seqs,
                                    groups or [0, len(seqs)])
        assert prefix.tolist() == want
    one = all(n == 1 for n in nq) and kw.get("max_q") is None
    kw = dict(kw, cu_q=None if one else i32(0, *np.cumsum(nq).tolist()), max_q=1 if one else kw.get("max_q") or max(nq))
    # attended together, or the test would be one of something else (60 queries of 40
    # heads a key/value head are not, for 2000 tokens)
    if kw.get("max_prefix") == 1 << 20 or (kw.get("max_prefix") == 2000 and q.shape[1] // m.H < 40):
        assert tq.tq_kv_attention_workspace_bytes(
            m.cache, len(nq), q.shape[1], n_tokens=q.shape[0], max_q=kw["max_q"], max_len=kw.get("max_len", 0),
            n_groups=1 if groups is None else len(groups) - 1, max_prefix=kw["max_prefix"]) > 0
    return tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda() if isinstance(q, np.ndarray) else q, seqs=seqs_t,
                              prefix=prefix, groups=g, out_f32=f32, want_lse=True, **kw)


@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64),
                                 (256, 128)])
@pytest.mark.parametrize("share", [1, 4, 7])
def test_decode(D, G, share):
    """One prompt, branches of one token and more, the prompt itself among them."""
    m = Branches([170], [0] * 11, [1, 2, 31, 32, 33, 0, 64, 65, 100, 5, 1], 2, D, G, 32, seed=D + G)
    seqs = m.kids + [0]
    q = rows((12, 2 * share, D), 5)
    for hint in (FEW, MANY, {}):
        o, lse = run(m, q, [1] * 12, seqs, **hint)
        check(m, q, [1] * 12, o, lse, seqs=seqs)
    h, _ = run(m, q, [1] * 12, seqs, f32=False, **FEW)
    check(m, q, [1] * 12, h, lse, seqs=seqs, f32=False)


@pytest.mark.parametrize("D,G,H,share,ps", [(64, 32, 1, 14, 64), (128, 64, 2, 4, 32), (256, 64, 1, 3, 32),
                                            (128, 128, 1, 1, 128), (64, 64, 2, 40, 32)])
def test_groups_and_many_queries(D, G, H, share, ps):
    """Groups of several sizes, one of them alone; rows without queries, with more
    of them than tokens behind the prefix, slots outside the cache and empty ones,
    a row that shares less than its group."""
    m = Branches([200, 70, 333, 0, 31], [0, 0, 0, 2, 2, 1, 1, 1, 4, 4], [9, 40, 3, 1, 130, 20, 1, 7, 3, 40], H, D, G, ps,
                 seed=D + share)
    seqs = [5, 6, -1, 7, 8, 9, 3, 10, 11, 12, 13, 14, 99, 2]
    nq = [3, 40, 2, 0, 1, 60, 1, 1, 2, 7, 3, 1, 1, 5]
    groups = [0, 4, 7, 10, 10, 13, 14]
    q = rows((sum(nq), H * share, D), 6)
    for hint in (FEW, MANY, {}):
        o, lse = run(m, q, nq, seqs, groups, **hint)
        check(m, q, nq, o, lse, seqs=seqs)
    # rows whose prompts differ share nothing; queries past max_q are left alone
    lone = run(m, q, nq, seqs, [0, 14], **FEW)
    check(m, q, nq, *lone, seqs=seqs)
    o2 = torch.full_like(o, 9.0)
    o2, lse2 = run(m, q, nq, seqs, groups, max_q=3, o=o2, **FEW)
    check(m, q, nq, o2, lse2, seqs=seqs, max_q=3)
    past = np.concatenate([np.arange(n) >= 3 for n in nq])
    assert bool((o2.cpu()[past] == 9).all())


@pytest.mark.parametrize("D,G,prompts,kids,tails,nq,share", [
    (128, 64, [5000], 6, [1, 2, 3, 4, 5, 6], 1, 4),         # a long prefix in many parts
    (128, 128, [4100], 40, list(range(1, 41)), 1, 8),       # many tiles
    (64, 32, [3000, 2000], 7, [700, 1, 1, 1, 1, 1, 1], 3, 2),
    (128, 32, [1500], 3, [1200, 1, 900], 2, 1),             # what is behind is in parts, too
    (256, 64, [2100], 5, [3, 3, 3, 3, 3], 3, 7),
    (128, 64, [2048, 1024, 4096], 30, [17] * 30, 1, 4),
    (128, 64, [700], 70, [5] * 70, 1, 4),
    (64, 64, [900], 33, [5] * 33, 4, 8),
])
def test_long(D, G, prompts, kids, tails, nq, share):
    P = len(prompts)
    parents = [i * P // kids for i in range(kids)]
    m = Branches(prompts, parents, tails, 2, D, G, 64, seed=7)
    groups = [0] + [i for i in range(1, kids) if parents[i] != parents[i - 1]] + [kids]
    q = rows((kids * nq, 2 * share, D), 8)
    o, lse = run(m, q, [nq] * kids, m.kids, groups)
    check(m, q, [nq] * kids, o, lse, seqs=m.kids)
    for kw in (dict(max_len=max(prompts), max_prefix=max(prompts), max_tail=max(tails)), dict(max_len=1),
               dict(max_prefix=64, max_tail=2000), dict(max_prefix=1 << 20)):
        o2, lse2 = run(m, q, [nq] * kids, m.kids, groups, **kw)       # hints decide the speed only
        check(m, q, [nq] * kids, o2, lse2, seqs=m.kids)
    assert all(torch.equal(a, b) for a, b in zip(run(m, q, [nq] * kids, m.kids, groups), (o, lse)))


@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 33, 64, 95, 128, 150])
def test_any_part_of_what_is_shared(prefix):
    """A caller may share less than there is; whole records are."""
    m = Branches([150], [0, 0, 0], [1, 20, 60], 2, 128, 64, 32)
    q = rows((3, 8, 128), 9)
    if prefix > 128:                                         # past the pages that are shared: as many as are
        prefix = 128
    for hint in (FEW, MANY):
        o, lse = run(m, q, [1] * 3, m.kids, prefix=i32(*[prefix] * 3), **hint)
        check(m, q, [1] * 3, o, lse, seqs=m.kids)
        # one row keeps out
        o, lse = run(m, q, [1] * 3, m.kids, prefix=i32(0, prefix, prefix), **hint)
        check(m, q, [1] * 3, o, lse, seqs=m.kids)


def test_a_query_inside_the_prefix_sees_its_past_only():
    """Rows whose last tokens are shared ones: nothing was added behind the fork."""
    m = Branches([128], [0, 0, 0], [0, 0, 3], 1, 64, 32, 32)
    q = rows((61, 4, 64), 3)
    for hint in (FEW, MANY, {}):
        for nq in ([10, 7, 4], [20, 1, 40]):                  # few rows beside each other, and many
            n = sum(nq)
            o, lse = run(m, q[:n], nq, m.kids, **hint)
            check(m, q[:n], nq, o, lse, seqs=m.kids)


@pytest.mark.parametrize("D,G,H,share,prompt,tails,nq", [
    (64, 32, 1, 1, 64, [36, 0], [1, 80]),                   # 16 queries before the first token, beside one that sees all
    (128, 64, 2, 4, 64, [36, 0], [1, 65]),                  # one of them among rows that see tokens
    (64, 64, 1, 2, 40, [0, 0], [50, 50]),                   # tiles of nothing else
    (256, 64, 1, 3, 100, [0, 5, 900, 1], [140, 1, 2, 103]),
    (128, 128, 2, 1, 320, [1, 1, 1], [1, 322, 400]),
])
def test_queries_before_a_slots_first_token(D, G, H, share, prompt, tails, nq):
    """Rows with more queries than their slots hold tokens: the first of them see
    nothing, whatever the rows beside them in a tile see."""
    m = Branches([prompt], [0] * len(tails), tails, H, D, G, 32, seed=D + share)
    q = rows((sum(nq), H * share, D), 4)
    for hint in (FEW, MANY, {}):
        o, lse = run(m, q, nq, m.kids, **hint)
        check(m, q, nq, o, lse, seqs=m.kids)
    # those past max_q are left alone beside them (few queries of many tokens may be attended row by row)
    for most, hint in ((3, dict(max_prefix=1 << 19)), (max(nq) - 1, MANY)):
        o2 = torch.full_like(o, 9.0)
        o2, lse2 = run(m, q, nq, m.kids, max_q=most, o=o2, **hint)
        check(m, q, nq, o2, lse2, seqs=m.kids, max_q=most)
        past = np.concatenate([np.arange(n) >= most for n in nq])
        assert bool((o2.cpu()[past] == 9).all())


def test_positions_without_a_page_and_poison():
    """A page that the table lost is left out; NaN and infinities in pages that
    nobody names, and behind the rows, do not show; those that are seen do."""
    m = Branches([128], [0, 0], [5, 40], 1, 64, 64, 32)
    q = rows((2, 4, 64), 2)
    prefix = i32(128, 128)
    m.cache.pages[1:3, 1] = -1
    o, lse = run(m, q, [1, 1], m.kids, prefix=prefix, **FEW)
    keep = [np.r_[0:32, 64:n] for n in (133, 168)]
    for s, kp in zip((1, 2), keep):
        m.k[s], m.v[s] = m.k[s][kp], m.v[s][kp]
    check(m, q, [1, 1], o, lse, seqs=m.kids)
    assert tq.tq_kv_shared_prefix(m.cache, seqs=i32(1, 2)).tolist() == [32, 32]
    bad = torch.full((1, 1, 64), float("nan"), dtype=torch.float16, device="cuda")
    m.cache.lens[0] = 128
    tq.tq_kv_append(m.cache, 0, bad, bad, i32(70), seqs=i32(0))        # a shared page
    o2, _ = run(m, q, [1, 1], m.kids, prefix=prefix, **FEW)
    assert bool(torch.isnan(o2).any(-1).all())


def test_a_window_attends_row_by_row():
    m = Branches([300], [0, 0, 0], [1, 20, 60], 2, 128, 64, 32)
    q = rows((3, 8, 128), 9)
    for kw in (dict(window=50), dict(window=50, sinks=7)):
        a = run(m, q, [1] * 3, m.kids, **kw)
        b = tq.tq_kv_attention(m.cache, 0, torch.from_numpy(q).cuda(), seqs=i32(*m.kids), out_f32=True, want_lse=True, **kw)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        check(m, q, [1] * 3, *a, seqs=m.kids, **kw)


def test_layers_strides_and_a_pool_past_4_gib():
    """The second layer, its pages beyond 4 GiB; queries inside a projection's output."""
    pb = 8 * 32 * 32 * (128 + 8)
    n = (5 << 30) // pb
    c = tq.KVCache.empty(2, n, 3, 4, 8, 128, 1024, 128)
    c.refs[:n - 5] = 1
    starts = tq.tq_kv_extend(c, cu_new=i32(0, 2050), seqs=i32(0))
    k, v = (rows((2050, 8, 128), 30 + i) for i in range(2))
    from oracle import q4
    tq.tq_kv_append(c, 1, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), starts, seqs=i32(0), cu_new=i32(0, 2050),
                    max_new=2050)
    tq.tq_kv_fork(c, i32(0, 0), i32(1, 2))
    m = Branches.__new__(Branches)
    m.H, m.D, m.G, m.ps, m.cache = 8, 128, 128, 1024, c
    m.k, m.v = ([q4.values(*q4.quantise(x, 128), 128)] * 3 for x in (k, v))
    assert tq.tq_kv_shared_prefix(c).tolist() == [2048] * 3
    q = rows((3, 32, 128), 3)
    buf = torch.zeros((3, 48, 130), dtype=torch.float16, device="cuda")
    view = buf[:, 3:35, 1:129]
    view.copy_(torch.from_numpy(q))
    for hint in (FEW, MANY, {}):
        o, lse = tq.tq_kv_attention(c, 1, view, prefix=tq.tq_kv_shared_prefix(c), out_f32=True, want_lse=True, **hint)
        check(m, q, [1] * 3, o, lse)


def test_workspaces_streams_and_graphs():
    m = Branches([3000], [0] * 12, [9] * 12, 2, 128, 64, 64)
    seqs, q = i32(*m.kids), torch.randn((12, 8, 128), dtype=torch.float16, device="cuda")
    prefix = tq.tq_kv_shared_prefix(m.cache, seqs=seqs)
    kw = dict(seqs=seqs, max_prefix=3000, max_tail=9, max_len=3009)
    call = lambda **more: tq.tq_kv_attention(m.cache, 0, q, prefix=prefix, **kw, **more)
    need = tq.tq_kv_attention_workspace_bytes(m.cache, 12, 8, max_len=3009, n_groups=1, max_prefix=3000, max_tail=9)
    want = call()
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:tq.WORKSPACE_COUNT_BYTES] = 0
    for _ in range(3):
        assert torch.equal(call(workspace=ws), want)
        assert bool((ws[:tq.WORKSPACE_COUNT_BYTES] == 0).all())
    with pytest.raises(tq.TqError):
        call(workspace=ws[:need - 16].clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p2 = tq.tq_kv_shared_prefix(m.cache, seqs=seqs)
        assert torch.equal(tq.tq_kv_attention(m.cache, 0, q, prefix=p2, **kw), want)
    torch.cuda.current_stream().wait_stream(side)
    # Two captured steps on one stream, their workspaces their own: room for a token, its
    # key and value, what is shared, attention; replayed in turn.
    new = [torch.randn((12, 2, 128), dtype=torch.float16, device="cuda") for _ in range(2)]
    outs = [torch.empty_like(want) for _ in range(2)]
    pre = torch.empty(12, dtype=torch.int32, device="cuda")

    def step(o):
        starts = tq.tq_kv_extend(m.cache, seqs=seqs)
        tq.tq_kv_append(m.cache, 0, *new, starts, seqs=seqs)
        tq.tq_kv_shared_prefix(m.cache, seqs=seqs, prefix=pre)
        return tq.tq_kv_attention(m.cache, 0, q, prefix=pre, o=o, **kw)

    saved = [t.clone() for t in m.cache._buffers()]

    def restore():
        for t, s in zip(m.cache._buffers(), saved):
            t.copy_(s)

    def inputs(i):
        g = torch.Generator(device="cuda").manual_seed(i)
        for x in (*new, q):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))

    step(outs[0])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, o in zip(graphs, outs):
        with torch.cuda.graph(g):
            step(o)
    restore()
    eager = []
    for i in range(6):
        inputs(i)
        step(outs[0])
        eager.append(outs[0].clone())
    restore()
    for i in range(6):
        inputs(i)
        outs[i % 2].zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], eager[i]), i
        call()                                                # the handle's own buffer is used in between


def test_prefixes_of_many_rows_and_pages():
    r = np.random.default_rng(0)
    c = tq.KVCache.empty(1, 5000, 40, 700, 1, 64, 32, 64)
    pages = np.full((40, 700), -1, np.int32)
    lens = np.zeros(40, np.int32)
    base = r.permutation(5000)[:700].astype(np.int32)
    for s in range(40):
        n = int(r.integers(0, 701))
        lens[s] = n * 32 - (int(r.integers(0, 32)) if n else 0)
        pages[s, :n] = base[:n]
        cut = int(r.integers(0, 1400))
        if cut < n:
            pages[s, cut] = r.integers(0, 5000)
    pages[7, 3], pages[8, 2], lens[9], lens[10] = -1, 10 ** 6, 10 ** 6, -4
    c.pages.copy_(torch.from_numpy(pages))
    c.lens.copy_(torch.from_numpy(lens))
    for trial in range(6):
        n = [1, 2, 40, 333, 64, 200][trial]
        seqs = r.integers(-1, 42, n).tolist()
        cuts = np.sort(r.integers(0, n + 1, int(r.integers(0, 6)) if n > 1 else 0)).tolist()
        groups = [0, *cuts, n]
        got = tq.tq_kv_shared_prefix(c, groups=i32(*groups) if n >= len(groups) - 1 else None, seqs=i32(*seqs))
        if n < len(groups) - 1:
            groups = [0, n]
        assert got.tolist() == decode.shared_prefix(pages.tolist(), lens.tolist(), 32, 5000, seqs, groups), trial
    # rows that no group has
    got = tq.tq_kv_shared_prefix(c, groups=i32(3, 30), seqs=None)
    assert got.tolist() == decode.shared_prefix(pages.tolist(), lens.tolist(), 32, 5000, list(range(40)), [3, 30])


@pytest.mark.parametrize("n_groups,most", [(64, 30), (65, 9), (130, 5), (4300, 3)])
def test_many_groups(n_groups, most):
    """More groups than a wave has lanes, some of them empty, rows without queries and
    with several; rows of one slot share its first tokens."""
    m = Branches([40, 100, 64], [], [], 1, 64, 32, 32)
    r = np.random.default_rng(n_groups)
    sizes = r.integers(0, most + 1, n_groups)
    sizes[[0, -1]] = 2
    groups = [0, *np.cumsum(sizes).tolist()]
    seqs = np.repeat(r.integers(0, 3, n_groups), sizes).tolist()
    nq = r.integers(0, 4, len(seqs)).tolist()
    q = rows((sum(nq), 3, 64), 8)
    prefix = np.repeat(np.where(sizes > 1, [[32], [96]], 0)[r.integers(0, 2, n_groups), np.arange(n_groups)], sizes)
    prefix = np.minimum(prefix, np.array([40, 100, 64])[seqs])
    o, lse = run(m, q, nq, seqs, groups, prefix=i32(*prefix.tolist()), **FEW)
    assert bool(torch.isfinite(o).all())
    some = sorted(set(r.integers(0, len(seqs), 60).tolist()) | {0, len(seqs) - 1})
    starts = np.concatenate([[0], np.cumsum(nq)])
    at = np.concatenate([np.arange(starts[i], starts[i + 1]) for i in some]).astype(np.int64)
    check(m, q[at], [nq[i] for i in some], o[at], lse[at], seqs=[seqs[i] for i in some])


@pytest.mark.parametrize("rows_", [2, 9, 40])
def test_prefixes_that_end_in_several_places(rows_):
    """Behind the first pages looked at, every row names another one somewhere: the
    first of those places counts, whoever finds one first."""
    r = np.random.default_rng(rows_)
    c = tq.KVCache.empty(1, 5000, rows_, 1500, 1, 64, 32, 64)
    for _ in range(20):
        pages = np.tile(r.permutation(5000)[:1500].astype(np.int32), (rows_, 1))
        for s in range(1, rows_):
            at = int(r.integers(256, 1500))
            pages[s, at] = 4999 - pages[s, at]
        c.pages.copy_(torch.from_numpy(pages))
        c.lens.fill_(1500 * 32)
        got = tq.tq_kv_shared_prefix(c)
        assert got.tolist() == [32 * int((pages != pages[0]).any(0).argmax())] * rows_


def test_refusals():
    m = Branches([100], [0, 0], [3, 3], 1, 64, 64, 32)
    q = torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
    seqs, pre = i32(*m.kids), i32(96, 96)
    call = lambda **kw: tq.tq_kv_attention(m.cache, 0, q, **dict(dict(seqs=seqs, prefix=pre), **kw))
    call()
    for kw in (dict(prefix=None, groups=i32(0, 2)), dict(prefix=pre.float()), dict(prefix=pre[:1]), dict(prefix=pre.cpu()),
               dict(groups=i32(0, 2).long()), dict(max_prefix=1 << 32)):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(groups=i32(0, 1, 1, 2)), dict(max_prefix=-1), dict(max_tail=-1), dict(sinks=-1)):
        with pytest.raises(tq.TqError) as e:
            call(**kw)
        assert e.value.status == 2, kw
    with pytest.raises(tq.TqError) as e:
        call(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), **FEW)
    assert e.value.status == 2
    for kw in (dict(groups=i32(0, 1, 1, 2), seqs=seqs), dict(seqs=torch.zeros(70000, dtype=torch.int32, device="cuda"))):
        with pytest.raises(tq.TqError) as e:
            tq.tq_kv_shared_prefix(m.cache, **kw)
        assert e.value.status == 2, kw
    with pytest.raises(ValueError):
        tq.tq_kv_shared_prefix(m.cache, seqs=seqs, prefix=i32(0))
