"""A decode step of branches of a prompt, its operators one after the other
(GPU): rotary positions of one projection's queries and keys, in place; the
keys and values into the cache; attention over the shared prefix in the first
layer, behind a window with sinks in the second; the output head; log
probabilities of the chosen tokens, the entropy and the most likely ones.
Every operator is checked against the fp64 oracle on what the one before it
gave (tolerances: where the operators' own tests derive them), and the whole
step, captured in two graphs, against the same calls outside of one, bit by bit.
"""

import numpy as np
import pytest
import torch

from kv_helpers import rows
from oracle import q4
from paper_2609_09240_amd import tq
from scope_helpers import Branches, check as check_attention, i32
from test_gpu_logprobs import check as check_logprobs
from test_gpu_rope import check as check_rope

pytestmark = pytest.mark.gpu

HQ, HKV, D, G, PS, V = 8, 2, 128, 64, 32, 3001
WINDOW, SINKS = 70, 5


class Step:
    """The buffers of a step of 12 branches and its calls."""

    def __init__(self, seed):
        self.m = Branches([1000], [0] * 12, [1, 2, 30, 31, 32, 33, 5, 64, 70, 9, 100, 4], HKV, D, G, PS, seed=seed, n_layers=2)
        c = self.m.cache
        c.data[1].copy_(c.data[0])                             # the second layer holds the same tokens
        self.seqs = i32(*self.m.kids)
        B = len(self.m.kids)
        self.rows = B
        self.proj = [torch.empty((B, (HQ + 2 * HKV) * D), dtype=torch.float16, device="cuda") for _ in range(2)]
        self.ids = torch.zeros((B, 2), dtype=torch.int32, device="cuda")
        # pairs of three axes in sections, as for images and video
        self.axis = torch.tensor([0] * 16 + [1] * 24 + [2] * 24, dtype=torch.uint8, device="cuda")
        self.pos = torch.empty((3, B), dtype=torch.int32, device="cuda")
        self.freq = (10000.0 ** (-torch.arange(64, device="cuda") / 64)).float()
        self.head = tq.tq_q4_quantize(torch.from_numpy(rows((V, HQ * D), 3)).cuda(), group=64)
        self.prefix = tq.tq_kv_shared_prefix(c, seqs=self.seqs)
        self.outs = {}

    def fill(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for p in self.proj:
            p.copy_(torch.randn(p.shape, generator=g, device="cuda"))
        self.ids.copy_(torch.randint(0, V, self.ids.shape, generator=g, device="cuda"))

    def parts(self, i):
        p = self.proj[i].view(self.rows, HQ + 2 * HKV, D)
        return p[:, :HQ], p[:, HQ:HQ + HKV], p[:, HQ + HKV:]

    def run(self, workspaces=None):
        ws = workspaces or (None, None, None)
        starts = tq.tq_kv_extend(self.m.cache, seqs=self.seqs)
        self.pos[0].copy_(starts)
        self.pos[1].copy_(starts // 7)
        self.pos[2].copy_(starts % 7)
        o = []
        for i in range(2):
            q, k, v = self.parts(i)
            tq.tq_rope(q, k, self.pos, self.freq, axis=self.axis, q_out=q, k_out=k)
            tq.tq_kv_append(self.m.cache, i, k, v, starts, seqs=self.seqs)
            kw = dict(prefix=self.prefix, max_prefix=1 << 20) if i == 0 else dict(window=WINDOW, sinks=SINKS)
            o.append(tq.tq_kv_attention(self.m.cache, i, q, seqs=self.seqs, workspace=ws[i], want_lse=True, **kw))
        x = torch.cat([t[0].view(self.rows, HQ * D) for t in o])
        logits = tq.tq_q4_gemm(self.head, x, out_f32=True)
        return o, logits, tq.tq_logprobs(logits, torch.cat([self.ids, self.ids]), top=5, scale=0.03, want_entropy=True,
                                         workspace=ws[2])


def test_every_operator_on_what_the_one_before_gave():
    s = Step(1)
    m = s.m
    s.fill(2)
    before = [[t.clone() for t in s.parts(i)] for i in range(2)]
    assert s.prefix.tolist() == [992] * 12   # the prompt's full pages
    o, logits, got = s.run()
    pos = s.pos.cpu().numpy()
    assert pos[0].tolist() == [1000 + t for t in [1, 2, 30, 31, 32, 33, 5, 64, 70, 9, 100, 4]]
    assert m.cache.lens.tolist() == [1000] + [p + 1 for p in pos[0].tolist()]
    held = list(m.k), list(m.v)
    for i in range(2):
        q, k, v = s.parts(i)
        for x, y in zip(before[i], (q, k)):
            check_rope(y, x.cpu().numpy(), pos, s.freq.cpu().numpy(), s.axis.cpu().numpy())
        assert torch.equal(v, before[i][2])
        m.k, m.v = list(held[0]), list(held[1])
        for new, mine in ((k, m.k), (v, m.v)):
            values = q4.values(*q4.quantise(new.cpu().numpy(), G), G)
            for b, slot in enumerate(m.kids):
                mine[slot] = np.concatenate([mine[slot], values[b:b + 1]])
        kw = {} if i == 0 else dict(window=WINDOW, sinks=SINKS)
        check_attention(m, q.cpu().numpy(), [1] * 12, *o[i], seqs=m.kids, f32=False, **kw)
    x = torch.cat([t[0].view(12, HQ * D) for t in o]).cpu().numpy().astype(np.float64)
    w = tq.tq_q4_unpack_fp16(s.head).cpu().numpy().astype(np.float64)
    # exact products, sums of HQ D terms in fp32; weights that were rounded to fp16
    bound = (np.abs(x) @ np.abs(w).T) * (2.0 ** -11 + HQ * D * 2.0 ** -24) + 1e-6
    assert (np.abs(logits.cpu().numpy() - x @ w.T) <= bound).all()
    check_logprobs(logits.cpu().numpy(), got, torch.cat([s.ids, s.ids]).cpu().numpy(), 5, 0.03)


def flat(r):
    o, logits, lp = r
    return [t for pair in o for t in pair] + [logits, *lp]


def test_two_captured_steps_give_what_the_calls_give():
    s = Step(4)
    c = s.m.cache
    sizes = (tq.tq_kv_attention_workspace_bytes(c, 12, HQ, n_groups=1, max_prefix=1 << 20),
             tq.tq_kv_attention_workspace_bytes(c, 12, HQ, window=WINDOW, sinks=SINKS),
             tq.tq_logprobs_workspace_bytes(24, V, n_ids=2, n_top=5))
    saved = [t.clone() for t in c._buffers()]

    def restore():
        for t, x in zip(c._buffers(), saved):
            t.copy_(x)

    s.fill(0)
    s.run()
    torch.cuda.synchronize()
    # Both graphs share their workspaces: replays on one stream do not overlap.
    ws = [torch.zeros(max(n, tq.WORKSPACE_COUNT_BYTES), dtype=torch.uint8, device="cuda") for n in sizes]
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(flat(s.run(ws)))
    restore()
    eager = []
    for i in range(6):
        s.fill(10 + i)
        eager.append([t.clone() for t in flat(s.run())])
    end = [t.clone() for t in c._buffers()]
    restore()
    for i in range(6):
        s.fill(10 + i)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(outs[i % 2], eager[i]):
            assert torch.equal(a, b), i
        tq.tq_logprobs(torch.randn((3, 9000), device="cuda"), top=20)   # eager work in between
        tq.tq_kv_attention(c, 0, s.parts(0)[0], seqs=s.seqs, prefix=s.prefix, max_prefix=1 << 20)
    for a, b in zip(c._buffers()[1:], end[1:]):
        assert torch.equal(a, b)


def test_scales_that_32_bits_do_not_hold_are_refused():
    s = Step(6)
    s.fill(1)
    q = s.parts(0)[0]
    for scale in (1e39, -1e39, float("inf"), float("nan")):
        for call in (lambda: tq.tq_rope(q, None, s.pos[0].zero_(), s.freq, scale=scale),
                     lambda: tq.tq_logprobs(s.freq.view(1, 64), top=1, scale=scale),
                     lambda: tq.tq_kv_attention(s.m.cache, 0, q, seqs=s.seqs, scale=scale),
                     lambda: tq.tq_kv_attention(s.m.cache, 0, q, seqs=s.seqs, scale=scale, window=9, sinks=1)):
            with pytest.raises(tq.TqError):
                call()


def test_tensors_of_another_device_are_refused(monkeypatch):
    s = Step(5)
    s.fill(1)
    q = s.parts(0)[0]
    calls = (lambda: tq.tq_rope(q, None, s.pos[0].zero_(), s.freq), lambda: tq.tq_logprobs(s.freq.view(1, 64), top=1),
             lambda: tq.tq_kv_shared_prefix(s.m.cache, seqs=s.seqs),
             lambda: tq.tq_kv_attention(s.m.cache, 0, q, seqs=s.seqs, prefix=s.prefix),
             lambda: tq.tq_kv_attention(s.m.cache, 0, q, seqs=s.seqs, window=9, sinks=1))
    for call in calls:
        call()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
