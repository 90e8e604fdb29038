"""Ragged calls of the 4-bit cache that do not say how many tokens a row has at
most (GPU): every token of the call is written, read and computed."""

import pytest
import torch

from kv_helpers import Model, rows
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu


def _i(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_append_and_read_take_every_token():
    c = tq.KVCache.empty(1, 12, 3, 5, 2, 64, 32, 32)
    new = _i(0, 70, 70, 103)
    starts = tq.tq_kv_extend(c, cu_new=new)
    k, v = (torch.from_numpy(rows((103, 2, 64), i)).cuda() for i in (1, 2))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    tq.tq_kv_append(c, 0, k, v, starts, cu_new=new, d_err=err)
    assert int(err) == 0
    want = tq.tq_kv_read(c, 0, starts, 103, cu_new=new, max_new=70)
    for t in (c.data, *want):
        assert t.numel() > 0
    other = tq.KVCache.empty(1, 12, 3, 5, 2, 64, 32, 32)
    starts = tq.tq_kv_extend(other, cu_new=new)
    tq.tq_kv_append(other, 0, k, v, starts, cu_new=new, max_new=70)
    got = [torch.full_like(k, 9.0) for _ in range(2)]
    tq.tq_kv_read(other, 0, starts, 103, cu_new=new, k=got[0], v=got[1])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("lens,nq", [([90, 70, 5], [13, 70, 1]), ([1, 2000, 300], [1, 30, 0])])
def test_attention_computes_every_query(lens, nq):
    m = Model(lens, 2, 64, 32, 32)
    q = torch.from_numpy(rows((sum(nq), 8, 64), 3)).cuda()
    cu = _i(0, *torch.tensor(nq).cumsum(0).tolist())
    # The number only decides how the work is laid out: a workgroup a tile, or
    # parts that are joined, whose fp32 sums differ in their order.
    want = tq.tq_kv_attention(m.cache, 0, q, cu_q=cu, max_q=max(nq), out_f32=True)
    got = torch.full_like(want, 9.0)
    lse = torch.full(want.shape[:2], 9.0, device="cuda")
    tq.tq_kv_attention(m.cache, 0, q, cu_q=cu, o=got, lse=lse, out_f32=True)
    assert float((got - want).abs().max()) <= 1e-4 and bool((lse != 9.0).all())


def test_a_given_number_still_holds():
    m = Model([50, 40], 1, 64, 64, 32)
    q = torch.from_numpy(rows((8, 2, 64), 3)).cuda()
    o = torch.full((8, 2, 64), 9.0, dtype=torch.float16, device="cuda")
    tq.tq_kv_attention(m.cache, 0, q, cu_q=_i(0, 5, 8), max_q=2, o=o)
    assert bool((o[2:5] == 9).all()) and bool((o[7:] == 9).all()) and bool((o[[0, 1, 5, 6]] != 9).any(-1).all())
