"""Numbers that do not fit the library's 32-bit arguments are refused by the
4-bit cache's calls, not cut to their low bits (GPU)."""

import pytest
import torch

from kv_helpers import Model, rows
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu

WIDE = (1 << 31, 1 << 32, (1 << 32) + 1, (1 << 63), -(1 << 31) - 1, -(1 << 32), -(1 << 32) + 5)


@pytest.mark.parametrize("x", WIDE)
def test_wide_numbers_are_refused(x):
    m = Model([70], 1, 64, 64, 32)
    q = torch.from_numpy(rows((1, 2, 64), 1)).cuda()
    k = q[:, :1].contiguous()
    cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = m.cache.data.clone()
    for kw in (dict(layer=x), dict(window=x), dict(max_len=x), dict(max_q=x, cu_q=cu)):
        with pytest.raises(ValueError):
            tq.tq_kv_attention(m.cache, **dict(dict(layer=0, q=q), **kw))
    for kw in (dict(layer=x), dict(max_new=x, cu_new=cu)):
        with pytest.raises(ValueError):
            tq.tq_kv_append(m.cache, **dict(dict(layer=0, k=k, v=k, starts=at), **kw))
        with pytest.raises(ValueError):
            tq.tq_kv_read(m.cache, **dict(dict(layer=0, starts=at, n_tokens=1), **kw))
    assert torch.equal(m.cache.data, before)


def test_the_largest_numbers_are_taken():
    m = Model([70], 1, 64, 64, 32)
    q = torch.from_numpy(rows((1, 2, 64), 1)).cuda()
    most = (1 << 31) - 1
    want = tq.tq_kv_attention(m.cache, 0, q, out_f32=True)
    # the same layout of the work: none of these splits 70 tokens
    assert torch.equal(tq.tq_kv_attention(m.cache, 0, q, out_f32=True, window=most), want)
    assert torch.equal(tq.tq_kv_attention(m.cache, 0, q, out_f32=True, max_q=most), want)
