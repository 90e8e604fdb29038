"""A decode loop on the library: ternary projections, a key/value cache held
in 4 bits, and a 4-bit output head.

    python examples/decode.py [--layers 2] [--branches 3] [--tokens 24]

A small decoder with random weights (RMS norm, rotary positions, grouped
heads, SwiGLU) reads a prompt, is forked into branches that share the
prompt's pages, decodes each of them for a while (the pages that they share are
attended once for all of them), keeps the most likely one, gives the others'
pages back, compacts the pool and goes on, at one row, from a HIP graph.  The
projections are quantised by ``quantize_linear``; norms and the activation are a
few lines of torch.
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_09240_amd import tq  # noqa: E402


class Decoder:
    """Weights and cache of a small decoder, and one step of it."""

    def __init__(self, hidden=1024, heads=8, kv_heads=2, head_dim=128, inter=2048, vocab=5000, layers=2, slots=8,
                 pages=64, page_size=32, max_pages=16, group=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).to(torch.float16)

        self.heads, self.kv_heads, self.d, self.vocab = heads, kv_heads, head_dim, vocab
        self.embed = torch.randn((vocab, hidden), generator=g, device="cuda").to(torch.float16)
        self.layers = [{name: tq.quantize_linear(weight(n, k)) for name, n, k in (
            ("q", heads * head_dim, hidden), ("k", kv_heads * head_dim, hidden), ("v", kv_heads * head_dim, hidden),
            ("o", hidden, heads * head_dim), ("gate", inter, hidden), ("up", inter, hidden), ("down", hidden, inter))}
            for _ in range(layers)]
        self.head = tq.tq_q4_quantize(weight(vocab, hidden), group=64)
        self.cache = tq.KVCache.empty(layers, pages, slots, max_pages, kv_heads, head_dim, page_size, group)
        self.max_len = max_pages * page_size
        self.freq = 10000.0 ** (-torch.arange(0, head_dim, 2, device="cuda") / head_dim)

    @staticmethod
    def norm(x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(torch.float16)

    @staticmethod
    def project(mats, x):
        """x W^T for matrices that read the same x [T, K]."""
        if x.shape[0] == 1:
            return [y.unsqueeze(0) for y in tq.tq_gemv_grouped(mats, x[0])]
        return [tq.tq_gemm_smallbatch(m, x) for m in mats]

    def layer(self, w, i, x, pos, q_of, starts, seqs, cu, max_new):
        """One decoder layer on x [T, hidden]; q_of attends: (layer, q) -> o."""
        T = x.shape[0]
        q, k, v = self.project([w["q"], w["k"], w["v"]], self.norm(x))
        q, k = q.view(T, self.heads, self.d), k.view(T, self.kv_heads, self.d)
        tq.tq_rope(q, k, pos, self.freq, q_out=q, k_out=k)
        tq.tq_kv_append(self.cache, i, k, v.view(T, self.kv_heads, self.d), starts, seqs=seqs, cu_new=cu,
                        max_new=max_new)
        x = x + self.project([w["o"]], q_of(i, q).view(T, -1))[0]
        gate, up = self.project([w["gate"], w["up"]], self.norm(x))
        act = (torch.nn.functional.silu(gate.float()) * up.float()).to(torch.float16)
        return x + self.project([w["down"]], act)[0]

    def step(self, tokens, seqs, new=None, workspace=None, prefix=None):
        """Logits [rows, vocab] after new tokens [T] of slots `seqs`: one token a
        row, or new[i] of them (a list).  T is at most 64.  prefix: the first
        tokens that the slots have in the same pages."""
        rows = seqs.numel()
        cu = None
        if new is not None:
            cu = torch.tensor([0, *torch.tensor(new).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
        starts = tq.tq_kv_extend(self.cache, cu_new=cu, seqs=seqs)
        pos = starts if cu is None else torch.cat(
            [starts[i] + torch.arange(n, dtype=torch.int32, device="cuda") for i, n in enumerate(new)])

        def attend(i, q):
            return tq.tq_kv_attention(self.cache, i, q, seqs=seqs, cu_q=cu, max_q=1 if new is None else max(new),
                                      max_len=self.max_len, workspace=workspace, prefix=prefix)

        x = self.embed[tokens]
        for i, w in enumerate(self.layers):
            x = self.layer(w, i, x, pos, attend, starts, seqs, cu, 1 if new is None else max(new))
        last = x if cu is None else x[cu[1:].long() - 1]
        assert last.shape[0] == rows
        return tq.tq_q4_gemm(self.head, self.norm(last), out_f32=True)


def slots(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def generate(layers=2, branches=3, tokens=24, seed=0, log=print):
    """Runs the loop; returns the tokens of the branch that was kept and its
    decoder."""
    m = Decoder(layers=layers, slots=branches + 1, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    prompt = torch.randint(0, m.vocab, (45,), generator=g, device="cuda")
    logits = m.step(prompt, slots(0), new=[45])
    log(f"prompt: 45 tokens in {int((m.cache.refs > 0).sum())} pages of {m.cache.page_size}")

    # Branches share the prompt's full pages; each starts with another token.
    kids = slots(*range(1, branches + 1))
    tq.tq_kv_fork(m.cache, slots(*[0] * branches), kids)
    tq.tq_kv_free(m.cache, slots(0))
    log(f"{branches} branches: {int((m.cache.refs > 0).sum())} pages, {int((m.cache.refs > 1).sum())} of them shared")
    shared = tq.tq_kv_shared_prefix(m.cache, seqs=kids)
    _, _, ids, logp = tq.tq_logprobs(logits, top=branches)
    nxt, logp = ids[0], logp[0]
    out = [[t] for t in nxt.tolist()]
    for _ in range(tokens // 2):
        logits = m.step(nxt, kids, prefix=shared)
        _, _, ids, best = tq.tq_logprobs(logits, top=1)
        nxt, logp = ids[:, 0], logp + best[:, 0]
        for o, t in zip(out, nxt.tolist()):
            o.append(t)

    # Keep the most likely branch.
    keep = int(logp.argmax())
    rest = [int(s) for i, s in enumerate(kids) if i != keep]
    if rest:
        tq.tq_kv_free(m.cache, slots(*rest))
    n_live = torch.zeros(1, dtype=torch.int32, device="cuda")
    tq.tq_kv_compact(m.cache, n_live=n_live)
    log(f"branch {keep} kept: {int(n_live)} pages at the front of the pool")

    # One row from here on: the step as a graph, its token and logits in place.
    seq, tok, kept = kids[keep:keep + 1].clone(), nxt[keep:keep + 1].clone(), out[keep]
    ws = m.cache.attention_workspace(tq.tq_kv_attention_workspace_bytes(m.cache, 1, m.heads, max_len=m.max_len))
    ws_top = torch.zeros(tq.tq_logprobs_workspace_bytes(1, m.vocab, n_ids=0, n_top=1), dtype=torch.uint8, device="cuda")

    def most_likely(logits):
        return tq.tq_logprobs(logits, top=1, workspace=ws_top)[2][0]

    left = tokens - tokens // 2
    # (A first step outside of the graph; it counts.)
    tok.copy_(most_likely(m.step(tok, seq, workspace=ws)))
    kept.append(int(tok))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        logits = m.step(tok, seq, workspace=ws)
        tok.copy_(most_likely(logits))
    for _ in range(left - 1):
        graph.replay()
        kept.append(int(tok))
    log(f"{len(kept)} tokens decoded, {int(m.cache.lens[int(seq)])} in the cache; {int((m.cache.refs > 0).sum())} pages")
    return prompt.tolist(), kept, m, int(seq), logits


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--branches", type=int, default=3)
    ap.add_argument("--tokens", type=int, default=24)
    a = ap.parse_args()
    _, kept, *_ = generate(a.layers, a.branches, a.tokens)
    print("tokens:", kept)
