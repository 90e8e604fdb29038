"""Workspaces of captured calls (GPU): a graph captured on the stream of the
warm-up, replayed after larger eager calls there, beside memory that was
allocated since, gives what the eager call gives."""

import numpy as np
import pytest
import torch

from kv_helpers import Model, rows
from oracle import q4
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu


def _replayed(small, large, inputs, out):
    """`small` and `large` run on the current stream; inputs(i) sets the i-th
    inputs, out is what small writes."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        inputs(0)
        small()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            small()
        held = []
        for i in range(1, 4):
            inputs(i)
            small()
            want = out.clone()
            large()
            held.append(torch.full((64 << 20,), 0x5A, dtype=torch.uint8, device="cuda"))   # where a freed buffer was
            out.zero_()
            g.replay()
            s.synchronize()
            assert torch.equal(out, want), i
            assert all(bool((t == 0x5A).all()) for t in held), i
    torch.cuda.current_stream().wait_stream(s)


def test_attention():
    m = Model([3000, 2500], 2, 128, 64, 64)
    many = Model([3000] * 12, 2, 128, 64, 64)
    q = torch.zeros((2, 8, 128), dtype=torch.float16, device="cuda")
    wide = torch.randn((12, 32, 128), device="cuda").half()
    o = torch.empty_like(q)
    _replayed(lambda: tq.tq_kv_attention(m.cache, 0, q, o=o, max_len=3000),
              # more parts in the handle's own buffer, and another handle's
              lambda: (tq.tq_kv_attention(m.cache, 0, wide[:2], max_len=3008),
                       tq.tq_kv_attention(many.cache, 0, wide, max_len=3000)),
              lambda i: q.copy_(torch.from_numpy(rows((2, 8, 128), i))), o)


def test_products():
    r = np.random.default_rng(0)
    w = torch.from_numpy((r.standard_normal((300, 4096)) * 0.02).astype(np.float16)).cuda()
    mat = tq.tq_q4_quantize(w, 64)
    x = torch.zeros((20, 4096), dtype=torch.float16, device="cuda")
    wide = torch.randn((64, 4096), device="cuda").half()
    y = torch.empty((20, 300), dtype=torch.float32, device="cuda")
    assert 0 < tq.tq_q4_workspace_bytes(mat, 20) < tq.tq_q4_workspace_bytes(mat, 64)
    _replayed(lambda: tq.tq_q4_gemm(mat, x, Y=y, out_f32=True), lambda: tq.tq_q4_gemm(mat, wide),
              lambda i: x.copy_(torch.from_numpy(rows((20, 4096), i))), y)


def test_only_the_counts_need_zeros():
    """Workspaces filled with anything behind their counts, call after call."""
    m = Model([3000, 40], 2, 128, 64, 64)
    q = torch.from_numpy(rows((2, 32, 128), 1)).cuda()
    want = tq.tq_kv_attention(m.cache, 0, q, out_f32=True)
    ws = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:tq.WORKSPACE_COUNT_BYTES] = 0
    for _ in range(3):
        assert torch.equal(tq.tq_kv_attention(m.cache, 0, q, out_f32=True, workspace=ws), want)
    codes = np.random.default_rng(1).integers(0, 16, (300, 4096)).astype(np.uint8)
    s, mn = (np.full((300, 64), v, np.float16) for v in (0.5, -3.0))
    cb, pb = q4.pack_matrix(codes, s, mn, 64)
    mat = tq.Q4Linear(300, 4096, 64, torch.from_numpy(cb).cuda(), torch.from_numpy(pb).cuda())
    x = np.random.default_rng(2).integers(-1, 2, (40, 4096)).astype(np.float16)
    ws = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:tq.WORKSPACE_COUNT_BYTES] = 0
    for _ in range(3):
        y = tq.tq_q4_gemm(mat, torch.from_numpy(x).cuda(), out_f32=True, workspace=ws)
        np.testing.assert_array_equal(y.cpu().numpy().astype(np.float64), q4.gemm(codes, s, mn, 64, x))


def test_one_workspace_for_products_and_attention():
    """The parts that one leaves are not the counts of the other."""
    m = Model([5000, 4000, 77], 2, 128, 64, 64)
    q = torch.from_numpy(rows((3, 32, 128), 1)).cuda()
    mat = tq.tq_q4_quantize(torch.randn((300, 8192), device="cuda").half(), 64)
    x = torch.randn((64, 8192), device="cuda").half()
    o, y = tq.tq_kv_attention(m.cache, 0, q), tq.tq_q4_gemm(mat, x)
    assert tq.tq_q4_workspace_bytes(mat, 64) > tq.WORKSPACE_COUNT_BYTES
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got_y = torch.full_like(y, 9.0)
        tq.tq_q4_gemm(mat, x, Y=got_y, workspace=ws)
        got_o = torch.full_like(o, 9.0)
        tq.tq_kv_attention(m.cache, 0, q, o=got_o, workspace=ws)
        assert torch.equal(got_y, y) and torch.equal(got_o, o)
        assert bool((ws[:tq.WORKSPACE_COUNT_BYTES] == 0).all())


@pytest.mark.parametrize("nq,max_len,window", [([1, 1], 0, 0), ([1, 1], 3000, 0), ([9, 2], 2000, 700), ([1, 1], 100, 0)])
def test_attention_workspace_bytes(nq, max_len, window):
    """What the size says is enough, and less is refused."""
    m = Model([3000, 40], 2, 128, 64, 64)
    q = torch.from_numpy(rows((sum(nq), 8, 128), 1)).cuda()
    cu = torch.tensor([0, *np.cumsum(nq).tolist()], dtype=torch.int32, device="cuda")
    kw = dict(cu_q=cu, max_q=max(nq), max_len=max_len, window=window)
    need = tq.tq_kv_attention_workspace_bytes(m.cache, 2, 8, sum(nq), max(nq), max_len, window)
    want = tq.tq_kv_attention(m.cache, 0, q, **kw)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    assert torch.equal(tq.tq_kv_attention(m.cache, 0, q, workspace=ws, **kw), want)
    assert (need == 0) == (max_len == 100)
    if need:
        with pytest.raises(tq.TqError):
            tq.tq_kv_attention(m.cache, 0, q, workspace=ws[:need - 16].clone(), **kw)
