"""The decode example end to end (GPU): the logits of its last step against
the same decoder in fp32 torch, with the dense weights that the packed ones
stand for and the keys and values that the cache holds.

Between the two lie roundings to fp16 in the example (about a dozen a layer,
each 2^-11 of a vector at most) and sums in another order: 2 layers and the
head make 26 of them, 1.3e-2 of the logits' norm if all added up.
"""

import os
import sys

import pytest
import torch

from paper_2609_09240_amd import tq

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_decode_example_against_dense_fp32():
    import decode
    said = []
    prompt, kept, m, seq, logits = decode.generate(layers=2, branches=3, tokens=24, log=said.append)
    text = prompt + kept
    n = len(text) - 1                                   # the last token has not been read yet
    assert len(kept) == 1 + 24 and int(m.cache.lens[seq]) == n
    assert "shared" in said[1] and int((m.cache.refs > 1).sum()) == 0
    live = int((m.cache.refs > 0).sum())
    assert live == -(-n // m.cache.page_size) and bool((m.cache.refs[live:] == 0).all())

    pos = torch.tensor([n - 1], device="cuda")
    x = m.embed[text[n - 1]].float()[None]

    def dense(mat):
        return tq.tq_unpack_fp16(mat).float()

    def norm(v):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6)

    row = torch.tensor([seq], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for i, w in enumerate(m.layers):
        h = norm(x)
        q = (h @ dense(w["q"]).t()).view(1, m.heads, m.d)
        a = (pos.float()[:, None] * m.freq)[:, None]
        q1, q2 = q.chunk(2, -1)
        q = torch.cat([q1 * torch.cos(a) - q2 * torch.sin(a), q2 * torch.cos(a) + q1 * torch.sin(a)], -1)[0]
        k, v = tq.tq_kv_read(m.cache, i, zero, n, seqs=row, cu_new=cu, max_new=n)
        share = m.heads // m.kv_heads
        o = []
        for head in range(m.heads):
            p = torch.softmax(k[:, head // share].float() @ q[head] * m.d ** -0.5, -1)
            o.append(p @ v[:, head // share].float())
        x = x + torch.cat(o)[None] @ dense(w["o"]).t()
        h = norm(x)
        act = torch.nn.functional.silu(h @ dense(w["gate"]).t()) * (h @ dense(w["up"]).t())
        x = x + act @ dense(w["down"]).t()
    want = norm(x) @ tq.tq_q4_unpack_fp16(m.head).float().t()
    assert float((logits - want).norm() / want.norm()) <= 1.3e-2
    assert kept[-1] == int(logits.argmax())
