"""Performance cases of the 4-bit operators around the ternary projections of
a decode step: the products with 4-bit weights, the key/value cache held in
4 bits, attention over it, and its pages.

A case is one of five kinds of work:

* ``q4``       B activation rows times a matrix of 4-bit weights with a scale
               and an offset per group (an output head, a projection kept at
               4 bits): ``tq_q4_gemm``;
* ``append``   new keys and values of one layer quantised into the pages of
               their sequences, and read back as fp16: ``tq_kv_append`` and
               ``tq_kv_read``;
* ``attn``     attention of new tokens over the pages: ``tq_kv_attention``;
* ``fork``     the step of a search that keeps several continuations: the
               branches that lost are freed and the winners forked anew:
               ``tq_kv_free`` and ``tq_kv_fork``;
* ``churn``    half of the sequences end, the pool is compacted and new ones
               come, then the same with the other half: ``tq_kv_free``,
               ``tq_kv_compact`` and ``tq_kv_extend``.

``own`` chooses between the library's calls and the plain form, which works
on the same packed bytes with elementary torch operations in 32 bits.

The packed layouts.  Eight 4-bit codes make a 32-bit word; element e of the
eight sits in nibble NIBBLE[e].  A matrix [N, K] is cut into tiles of 16
rows and 128 inputs of 1024 bytes, [N/16][K/128][c 4][row 16][j 4] words,
the word holding inputs 32 j + 8 c + e; its parameters are fp16 (scale,
offset) pairs [N/16][K/group][row 16].  A page holds, per key/value head,
page_size/32 records of 32 tokens: key words [half 2][c 4][token 16][D/32 j]
(channels 32 j + 8 c + e of token 16 half + t), value words [D/64][c 4]
[channel 16][4] (one channel of tokens 4 c + i in nibble i and 16 + 4 c + i
in nibble 4 + i), then the fp16 (scale, offset) pairs of the keys [D/group]
[token 32] and of the values.
"""

import math
import random

import torch

own = False

GROUP = 128
NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)      # element e of eight -> nibble of the word
ORDER = (0, 2, 4, 6, 1, 3, 5, 7)       # nibble -> element
HIDDEN, INTER, KV = 4096, 12288, 1024  # the decoder layer of the package's synthetic workloads
HQ, HKV, D = 32, 8, 128                # its heads


def listed():
    return [
        # The smallest product: a key/value-sized projection on one row, where
        # the launch counts.
        q4("q4 1024x4096 b1", KV, HIDDEN, 1, 128),
        # An output head over a large vocabulary for one token: bytes count.
        q4("q4 head 131072x4096 b1", 131072, HIDDEN, 1, 64),
        # A down projection for sixteen users.
        q4("q4 4096x12288 b16", HIDDEN, INTER, 16, 128),
        # Sizes that no tile divides, small groups, a few rows, fp32 outputs.
        q4("q4 2999x5000 b5 g32", 2999, 5000, 5, 32, f32=True),
        # The cache's part of one decoded token for 64 users: one row each.
        append("append 64x1", 64, 2000, 1),
        # A chunk of prompts for three users whose caches end inside a tile.
        append("append 3x2000 g32", 3, 2500, 2000, g=32),
        # One user, a short conversation: latency.
        attn("attn b1 len 45", 1, 45),
        # A serving batch of ragged lengths, an idle slot among them.
        attn("attn b32 to 8192", 32, 8192),
        # One user with a long document.
        attn("attn b1 len 131072", 1, 131072, g=128),
        # A prompt's chunk over what is cached, smaller heads, a sliding
        # window, fp32 outputs and their log-sum.
        attn("attn chunk 2x1000 d64", 2, 5000, nq=1000, hq=14, hkv=2, d=64, g=32, window=2048, f32=True),
        # Four prompts, fifteen branches each.
        fork("fork 60 of 4", 4, 15, 1500, 12),
        # Sixty-four users, half of them replaced.
        churn("churn 64", 64, 600, 8),
    ]


def q4(name, n, k, b, g, f32=False):
    return dict(name=name, kind="q4", n=n, k=k, b=b, g=g, f32=f32)


def append(name, b, maxlen, new, hkv=HKV, d=D, g=64, ps=64, mix=1):
    return dict(name=name, kind="append", b=b, maxlen=maxlen, new=new, hkv=hkv, d=d, g=g, ps=ps, mix=mix)


def attn(name, b, maxlen, nq=1, hq=HQ, hkv=HKV, d=D, g=64, ps=64, window=0, f32=False, mix=1):
    return dict(name=name, kind="attn", b=b, maxlen=maxlen, nq=nq, hq=hq, hkv=hkv, d=d, g=g, ps=ps, window=window,
                f32=f32, mix=mix)


def fork(name, prompts, branches, maxlen, layers, hkv=HKV, d=D, g=64, ps=64, mix=1):
    return dict(name=name, kind="fork", b=prompts, branches=branches, maxlen=maxlen, layers=layers, hkv=hkv, d=d, g=g,
                ps=ps, mix=mix)


def churn(name, b, maxlen, layers, hkv=HKV, d=D, g=64, ps=64, mix=1):
    return dict(name=name, kind="churn", b=b, maxlen=maxlen, layers=layers, hkv=hkv, d=d, g=g, ps=ps, mix=mix)


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["q4", "q4", "q4", "append", "append", "attn", "attn", "attn", "attn", "fork", "churn"])
    mix = rng.randrange(1, 1 << 20)
    d = rng.choice([64, 128, 128])
    g = rng.choice([v for v in (32, 64, 64, 128) if v <= d])
    ps = rng.choice([32, 64, 64, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    if kind == "q4":
        k = log_int(256, 16384)
        if rng.random() < 0.6:
            k = -(-k // GROUP) * GROUP
        n = log_int(100, min(131072, 131072 * HIDDEN // k))
        b = rng.choice([1, 1, 2, 4, 8, 16, log_int(1, 64), log_int(9, 64)])
        n = min(n, max(100, 131072 * HIDDEN * 4 // (k * (3 + b))))
        c = q4("", n, k, b, rng.choice([32, 64, 128, 128]), f32=rng.random() < 0.3)
    elif kind == "append":
        new = rng.choice([1, 1, log_int(2, 16), log_int(17, 2048)])
        b = log_int(1, max(1, min(128, 6000 // new)))
        c = append("", b, new + log_int(32, 4096), new, hkv, d, g, ps, mix)
    elif kind == "attn":
        nq = rng.choice([1, 1, 1, 1, log_int(2, 16), log_int(17, 1024)])
        share = rng.choice([1, 2, 4, 4, 7, 8, 16] if nq <= 16 else [1, 2, 4])
        b = log_int(1, 64 if nq == 1 else 8 if nq <= 16 else 2)
        most = (131072 if nq == 1 else 16384 if nq <= 16 else 5000) // (b if nq == 1 else 1)
        c = attn("", b, nq + log_int(30, most), nq, share * hkv, hkv, d, g, ps, rng.choice([0, 0, 0, log_int(64, 4096)]),
                 rng.random() < 0.3, mix)
    elif kind == "fork":
        c = fork("", log_int(1, 6), log_int(1, 15), log_int(40, 1500), rng.randint(1, 12), hkv, d, g, ps, mix)
    else:
        c = churn("", log_int(2, 64), log_int(40, 600), rng.randint(1, 8), hkv, d, g, ps, mix)
    c.pop("name", None)
    return c


# --------------------------------------------------------------------------
# Sizes of a case.
# --------------------------------------------------------------------------

def _lens(c):
    """Tokens in the cache of every sequence once this pass's are in it:
    spread over their logarithm, the longest first, one idle slot (no tokens)
    in a decoding batch of eight or more."""
    r = random.Random(c["mix"])
    new = c.get("nq", c.get("new", 1))
    hi = c["maxlen"]
    lo = max(new, hi // 16, 1)
    v = [hi] + [max(lo, min(hi, round(math.exp(r.uniform(math.log(lo), math.log(max(lo, hi)))))))
                for _ in range(c["b"] - 1)]
    if c["kind"] == "attn" and new == 1 and c["b"] >= 8:
        v[3] = 0
    return v


def _rec(c):
    """Bytes of one record: 32 tokens of one head, keys and values."""
    return 32 * (c["d"] + 8 * c["d"] // c["g"])


def _pages(n, ps):
    return -(-n // ps)


def work(c):
    per = c["d"] + 8 * c["d"] // c["g"] if "d" in c else 0     # bytes of a token and head, keys and values
    if c["kind"] == "q4":
        n, k, b = c["n"], c["k"], c["b"]
        return {"bytes": n * k // 2 + 4 * n * -(-k // c["g"]) + 2 * b * k + (4 if c["f32"] else 2) * b * n,
                "flops": 2 * b * n * k}
    if c["kind"] == "append":
        t = c["b"] * c["new"] * c["hkv"]
        # fp16 rows in, 4-bit rows out; those back in, fp16 rows out
        return {"bytes": t * (4 * c["d"] + per + per + 4 * c["d"]), "flops": t * c["d"] * 2 * 6}
    if c["kind"] == "attn":
        pairs = read = 0
        for ln in _lens(c):
            w = c["window"] or ln
            q = min(c["nq"], ln)
            if q:
                first = ln - q
                full = max(0, min(q, w - first - 1))             # queries whose window holds all of the past
                pairs += full * (first + 1) + full * (full - 1) // 2 + (q - full) * w
                read += min(ln, w + q - 1)
        rows = c["b"] * c["nq"] * c["hq"]
        return {"bytes": read * c["hkv"] * per + rows * c["d"] * (2 + (4 if c["f32"] else 2)) + rows * 4,
                "flops": 4 * pairs * c["hq"] * c["d"]}
    page = c["hkv"] * (c["ps"] // 32) * _rec(c) * c["layers"]
    if c["kind"] == "fork":
        moved = sum(1 for ln in _lens(c) if ln % c["ps"]) * c["branches"]
        return {"bytes": 2 * moved * page + 16 * sum(_pages(ln, c["ps"]) for ln in _lens(c)) * c["branches"], "flops": 0}
    # churn: every sequence's pages move once a pass (half of the pages at a time)
    moved = sum(_pages(ln, c["ps"]) for ln in _lens(c))
    half = [sum(_pages(ln, c["ps"]) for ln in _lens(c)[k::2]) for k in (0, 1)]
    return {"bytes": 2 * 2 * min(half) * page + 16 * moved, "flops": 0}


# --------------------------------------------------------------------------
# Inputs, from the seed alone.
# --------------------------------------------------------------------------

def _gen(*key):
    h = 0
    for k in key:
        h = (h * 1000003 + int(k) + 12345) % (1 << 62)
    g = torch.Generator(device="cuda")
    g.manual_seed(h)
    return g


def _quantise(x, g):
    """Codes (uint8, as x) and (scale, offset) fp16 [..., last/g, 2] of fp16
    x, groups of g along the last dimension (a short last group stands)."""
    last = x.shape[-1]
    n = -(-last // g)
    xf = x.float()
    if n * g != last:
        xf = torch.cat([xf, xf[..., -1:].expand(*xf.shape[:-1], n * g - last)], -1)
    xg = xf.unflatten(-1, (n, g))
    lo = xg.amin(-1, keepdim=True)
    s = ((xg.amax(-1, keepdim=True) - lo) / 15.0).half()
    sf = s.float()
    q = torch.where(sf > 0, torch.round((xg - lo) / sf).clamp(0, 15), torch.zeros_like(xg)).to(torch.uint8)
    return q.flatten(-2)[..., :last], torch.cat([s, lo.half()], -1)


def _nibbles(q):
    """uint8 codes [..., 8] (in nibble order) -> bytes [..., 4]."""
    return q[..., 0::2] | (q[..., 1::2] << 4)


def _pack_matrix(q):
    """codes [N, K] -> the packed matrix's code buffer."""
    n, k = q.shape
    nt, kb = -(-n // 16), -(-k // 128)
    full = torch.zeros((nt * 16, kb * 128), dtype=torch.uint8, device=q.device)
    full[:n, :k] = q
    e = full.view(nt, 16, kb, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)[..., list(ORDER)]
    return _nibbles(e).reshape(-1).contiguous()


def _pack_params(p, n, k, g):
    """pairs [N, K/g, 2] -> the packed matrix's parameter buffer."""
    nt, ng = -(-n // 16), 128 // g * -(-k // 128)
    full = torch.zeros((nt * 16, ng, 2), dtype=torch.float16, device=p.device)
    full[:n, :p.shape[1]] = p
    return full.view(nt, 16, ng, 2).permute(0, 2, 1, 3).reshape(-1).contiguous()


def _pack_pages(k, v, g):
    """fp16 keys and values [P, H, ps, D] -> bytes [P, page_bytes]."""
    P, H, ps, d = k.shape
    qk, pk = _quantise(k, g)
    qv, pv = _quantise(v, g)
    nb = ps // 32
    kb = qk.view(P, H, nb, 2, 16, d // 32, 4, 8).permute(0, 1, 2, 3, 6, 4, 5, 7)[..., list(ORDER)]
    # value words: tokens (half, c, i) of channel (load, jd, dl); nibble 4 half + i
    vb = qv.view(P, H, nb, 2, 4, 4, d // 64, 4, 16).permute(0, 1, 2, 6, 4, 8, 7, 3, 5).flatten(-2)
    parts = [_nibbles(kb).reshape(P, H, nb, -1), _nibbles(vb).reshape(P, H, nb, -1)]
    for p in (pk, pv):
        parts.append(p.view(P, H, nb, 32, d // g, 2).permute(0, 1, 2, 4, 3, 5).contiguous().view(torch.uint8)
                     .reshape(P, H, nb, -1))
    return torch.cat(parts, -1).reshape(P, -1)


def _rows(shape, g):
    """Keys or values: N(0, 1), a few channels larger, as projections give."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)
    x[..., 3::37] *= 4.0
    return x


def _table(c, seed, n_seqs, held, spare):
    """Page table [n_seqs, max_pages], lengths and counts for sequences that
    hold `held` tokens, their pages in random order over a pool that is
    `spare` pages larger."""
    ps = c["ps"]
    need = [_pages(h, ps) for h in held]
    total = sum(need) + spare
    order = torch.randperm(total, generator=_gen(seed, 7), device="cuda").to(torch.int32)
    mp = max(need + [1]) + 1
    pages = torch.full((n_seqs, mp), -1, dtype=torch.int32)
    at = 0
    cpu = order.cpu()
    for s, n in enumerate(need):
        pages[s, :n] = cpu[at:at + n]
        at += n
    refs = torch.zeros(total, dtype=torch.int32)
    refs[cpu[:at].long()] = 1
    lens = torch.tensor(list(held) + [0] * (n_seqs - len(held)), dtype=torch.int32)
    return pages.cuda(), lens.cuda(), refs.cuda(), total


def _pool(c, seed, total, layers):
    shape = (total, c["hkv"], c["ps"], c["d"])
    out = []
    for layer in range(layers):
        g = _gen(seed, 11, layer)
        out.append(_pack_pages(_rows(shape, g), _rows(shape, g), c["g"]))
    return torch.stack(out)


def prepare(c, seed):
    st = {"case": dict(c)}
    g = _gen(seed, 1)
    if c["kind"] == "q4":
        n, k = c["n"], c["k"]
        codes, pairs = [], []
        for r in range(0, n, 16384):                        # rows at a time: fp32 copies of a large head are not kept
            w = torch.randn((min(16384, n - r), k), generator=g, device="cuda", dtype=torch.float16) * 0.02
            q, p = _quantise(w, c["g"])
            codes.append(_pack_matrix(q))
            pairs.append(_pack_params(p, q.shape[0], k, c["g"]))
        st.update(codes=torch.cat(codes), params=torch.cat(pairs),
                  x=torch.randn((c["b"], k), generator=g, device="cuda", dtype=torch.float16))
        return st
    lens = _lens(c)
    b = c["b"]
    layers = c.get("layers", 1)
    if c["kind"] == "fork":
        n_seqs = b * (1 + c["branches"])
        pages, lens_t, refs, total = _table(c, seed, n_seqs, lens, b * c["branches"] + 3)
        parents = torch.arange(b, device="cuda", dtype=torch.int32).repeat_interleave(c["branches"])
        children = torch.arange(b, n_seqs, device="cuda", dtype=torch.int32)
        st.update(parents=parents, children=children)
    else:
        pages, lens_t, refs, total = _table(c, seed, b, lens, b + 5)
        if c["kind"] == "churn":
            st["halves"] = []
            for k in (0, 1):
                slots = torch.arange(k, b, 2, dtype=torch.int32)
                cu = torch.zeros(len(slots) + 1, dtype=torch.int32)
                cu[1:] = torch.tensor(lens[k::2], dtype=torch.int32).cumsum(0)
                st["halves"].append((slots.cuda(), cu.cuda()))
    st.update(pages=pages, lens=lens_t, refs=refs, data=_pool(c, seed, total, layers))
    if c["kind"] == "append":
        t = b * c["new"]
        st["k"], st["v"] = _rows((t, c["hkv"], c["d"]), g), _rows((t, c["hkv"], c["d"]), g)
        st["starts"] = lens_t - c["new"]
        st["cu"] = torch.arange(0, t + 1, c["new"], device="cuda", dtype=torch.int32)
    elif c["kind"] == "attn":
        st["q"] = torch.randn((b * c["nq"], c["hq"], c["d"]), generator=g, device="cuda", dtype=torch.float16)
        st["cu"] = torch.arange(0, b * c["nq"] + 1, c["nq"], device="cuda", dtype=torch.int32)
    return st


# --------------------------------------------------------------------------
# The plain form: the definitions in 32 bits, on the packed bytes.
# --------------------------------------------------------------------------

def _codes(b):
    """bytes [..., 4] -> codes [..., 8] in element order."""
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)[..., list(NIBBLE)]


def _dense(codes, params, n, k, g):
    nt, kb = -(-n // 16), -(-k // 128)
    q = _codes(codes.view(nt, kb, 4, 16, 4, 4)).permute(0, 3, 1, 4, 2, 5).reshape(nt * 16, kb * 128 // g, g)
    p = params.view(nt, kb * 128 // g, 16, 2).permute(0, 2, 1, 3).reshape(nt * 16, kb * 128 // g, 2).float()
    return (q.float() * p[..., :1] + p[..., 1:]).reshape(nt * 16, kb * 128)[:n, :k]


def _plain_q4(st, c):
    y = st["x"].float() @ _dense(st["codes"], st["params"], c["n"], c["k"], c["g"]).t()
    return y if c["f32"] else y.half()


def _plain_pages(raw, c):
    """page bytes [P, page_bytes] -> fp32 keys and values [P, H, ps, D]."""
    d, g, nb = c["d"], c["g"], c["ps"] // 32
    P, H = raw.shape[0], c["hkv"]
    raw = raw.view(P, H, nb, _rec(c))
    ck, cv = raw[..., :16 * d], raw[..., 16 * d:32 * d]
    qk = _codes(ck.reshape(P, H, nb, 2, 4, 16, d // 32, 4)).permute(0, 1, 2, 3, 5, 6, 4, 7).reshape(P, H, nb * 32, d // g, g)
    b = cv.reshape(P, H, nb, d // 64, 4, 16, 4, 4)
    q = torch.stack([b & 15, b >> 4], -1).reshape(P, H, nb, d // 64, 4, 16, 4, 2, 4)    # [load, c, dl, jd, half, i]
    qv = q.permute(0, 1, 2, 7, 4, 8, 3, 6, 5).reshape(P, H, nb * 32, d // g, g)
    out = []
    for q, at in ((qk, 32 * d), (qv, 32 * d + 128 * d // g)):
        p = raw[..., at:at + 128 * d // g].contiguous().view(torch.float16).view(P, H, nb, d // g, 32, 2)
        p = p.permute(0, 1, 2, 4, 3, 5).reshape(P, H, nb * 32, d // g, 2).float()
        out.append((q.float() * p[..., :1] + p[..., 1:]).flatten(-2))
    return out


def _plain_append(st, c):
    """The records that the new tokens touch are decoded to codes, the new
    ones put in, and the records put back."""
    d, g, ps, H, nb = c["d"], c["g"], c["ps"], c["hkv"], c["ps"] // 32
    b, new = c["b"], c["new"]
    pos = st["starts"].long()[:, None] + torch.arange(new, device="cuda")             # [b, new]
    page = st["pages"].long().gather(1, pos // ps)
    page, slot = page.reshape(-1), (pos % ps).reshape(-1)
    data = st["data"][0]
    touched, back = torch.unique(page, return_inverse=True)
    raw = data[touched].view(len(touched), H, nb, _rec(c))
    P = len(touched)
    qk, pk = _quantise(st["k"], g)
    qv, pv = _quantise(st["v"], g)
    ck = raw[..., :16 * d].reshape(P, H, nb, 2, 4, 16, d // 32, 4)
    ck = torch.stack([ck & 15, ck >> 4], -1).flatten(-2)[..., list(NIBBLE)].permute(0, 1, 2, 3, 5, 6, 4, 7)
    ck = ck.reshape(P, H, ps, d)
    ck[back, :, slot] = qk
    bv = raw[..., 16 * d:32 * d].reshape(P, H, nb, d // 64, 4, 16, 4, 4)
    cv = torch.stack([bv & 15, bv >> 4], -1).reshape(P, H, nb, d // 64, 4, 16, 4, 2, 4)
    cv = cv.permute(0, 1, 2, 7, 4, 8, 3, 6, 5).reshape(P, H, ps, d)
    cv[back, :, slot] = qv
    kb = ck.view(P, H, nb, 2, 16, d // 32, 4, 8).permute(0, 1, 2, 3, 6, 4, 5, 7)[..., list(ORDER)]
    vb = cv.view(P, H, nb, 2, 4, 4, d // 64, 4, 16).permute(0, 1, 2, 6, 4, 8, 7, 3, 5).flatten(-2)
    raw[..., :16 * d] = _nibbles(kb).reshape(P, H, nb, -1)
    raw[..., 16 * d:32 * d] = _nibbles(vb).reshape(P, H, nb, -1)
    vals = []
    for q, p, at in ((qk, pk, 32 * d), (qv, pv, 32 * d + 128 * d // g)):
        old = raw[..., at:at + 128 * d // g].contiguous().view(torch.float16).view(P, H, nb, d // g, 32, 2)
        old = old.permute(0, 1, 2, 4, 3, 5).reshape(P, H, ps, d // g, 2)
        old[back, :, slot] = p
        raw[..., at:at + 128 * d // g] = old.view(P, H, nb, 32, d // g, 2).permute(0, 1, 2, 4, 3, 5).contiguous() \
            .view(torch.uint8).reshape(P, H, nb, -1)
    data[touched] = raw.view(P, -1)
    k, v = _plain_pages(data[touched], c)
    for x in (k, v):
        vals.append(x[back, :, slot].half())
    return tuple(vals)


def _plain_attn(st, c):
    b, nq, hq, H, d = c["b"], c["nq"], c["hq"], c["hkv"], c["d"]
    ps, mp = c["ps"], _pages(c["maxlen"], c["ps"])
    pages = st["pages"][:, :mp].long().clamp(min=0)
    k, v = _plain_pages(st["data"][0][pages.reshape(-1)], c)                            # [b*mp, H, ps, d]
    k, v = (x.view(b, mp, H, ps, d).transpose(1, 2).reshape(b, H, mp * ps, d) for x in (k, v))
    lens = st["lens"].long()[:, None]
    j = torch.arange(mp * ps, device="cuda")
    pos = lens - nq + torch.arange(nq, device="cuda")                                   # [b, nq]
    see = (j <= pos[..., None]) & (j < lens[..., None])
    if c["window"]:
        see &= j > pos[..., None] - c["window"]
    q = st["q"].float().view(b, nq, H, hq // H, d).permute(0, 2, 3, 1, 4).reshape(b, H, hq // H * nq, d)
    s = (q @ k.transpose(2, 3).contiguous()) * (d ** -0.5)
    s = s.view(b, H, hq // H, nq, -1).masked_fill(~see[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - top.clamp(min=-1e30))
    l = e.sum(-1, keepdim=True)
    v = v.masked_fill(~(j < lens)[:, None, :, None], 0.0)
    o = (e.view(b, H, hq // H * nq, -1) @ v).view(b, H, hq // H, nq, d) / torch.where(l > 0, l, torch.ones_like(l))
    lse = (top + torch.log(l))[..., 0]
    o = o.permute(0, 3, 1, 2, 4).reshape(b * nq, hq, d)
    return (o if c["f32"] else o.half()), lse.permute(0, 3, 1, 2).reshape(b * nq, hq).contiguous()


def _plain_free(st, slots):
    rows = st["pages"][slots]
    st["refs"].index_add_(0, rows.clamp(min=0).flatten(), -(rows >= 0).int().flatten())
    st["pages"][slots] = -1
    st["lens"][slots] = 0


def _plain_fork(st, c):
    p, ch = st["parents"].long(), st["children"].long()
    _plain_free(st, ch)
    ln = st["lens"][p]
    full, part = ln // c["ps"], ln % c["ps"] > 0
    rows = st["pages"][p]
    col = torch.arange(rows.shape[1], device="cuda")
    share = col < full[:, None]
    last = rows.gather(1, full[:, None].long())[part][:, 0].long()
    st["refs"].index_add_(0, rows.clamp(min=0).flatten(), share.int().flatten())
    free = torch.nonzero(st["refs"] == 0)[:len(last), 0]
    rows = torch.where(share, rows, -1)
    rows[part, full[part].long()] = free.int()
    st["refs"][free] = 1
    st["pages"][ch] = rows
    st["lens"][ch] = ln
    st["data"][:, free] = st["data"][:, last]
    return st["pages"], st["lens"], st["refs"], st["data"]


def _plain_compact(st):
    refs, n = st["refs"], st["refs"].numel()
    live = refs > 0
    idx = torch.arange(n, device="cuda")
    nl = live.sum()
    hole, mover = torch.nonzero(~live & (idx < nl))[:, 0], torch.nonzero(live & (idx >= nl))[:, 0]
    st["data"][:, hole] = st["data"][:, mover]
    to = idx.int()
    to[mover] = hole.int()
    refs[hole] = refs[mover]
    refs[mover] = 0
    st["pages"].copy_(torch.where(st["pages"] >= 0, to[st["pages"].clamp(min=0).long()], -1))


def _plain_extend(st, c, slots, cu):
    n = cu[1:] - cu[:-1]
    lens = st["lens"][slots]
    have, want = -(-lens // c["ps"]), -(-(lens + n) // c["ps"])
    rows = st["pages"][slots]
    col = torch.arange(rows.shape[1], device="cuda")
    take = (col >= have[:, None]) & (col < want[:, None])
    free = torch.nonzero(st["refs"] == 0)[:int(take.sum()), 0]
    rows[take] = free.int()
    st["refs"][free] = 1
    st["pages"][slots] = rows
    st["lens"][slots] = lens + n


def _plain_churn(st, c):
    for slots, cu in st["halves"]:
        _plain_free(st, slots.long())
        _plain_compact(st)
        _plain_extend(st, c, slots.long(), cu)
    return st["pages"], st["lens"], st["refs"], st["data"]


# --------------------------------------------------------------------------
# The library's calls.
# --------------------------------------------------------------------------

def _handle(st, c):
    """The handle that a program makes once and keeps beside its buffers."""
    from paper_2609_09240_amd import tq
    if "handle" not in st:
        if c["kind"] == "q4":
            st["handle"] = tq.Q4Linear(c["n"], c["k"], c["g"], st["codes"], st["params"])
        else:
            st["handle"] = tq.KVCache(st["data"], st["pages"], st["lens"], st["refs"], n_kv_heads=c["hkv"],
                                      head_dim=c["d"], page_size=c["ps"], group=c["g"])
    return tq, st["handle"]


def _own(st, c):
    tq, h = _handle(st, c)
    if c["kind"] == "q4":
        return tq.tq_q4_gemm(h, st["x"], out_f32=c["f32"])
    if c["kind"] == "append":
        one = c["new"] == 1
        tq.tq_kv_append(h, 0, st["k"], st["v"], st["starts"], cu_new=None if one else st["cu"], max_new=c["new"])
        return tq.tq_kv_read(h, 0, st["starts"], c["b"] * c["new"], cu_new=None if one else st["cu"], max_new=c["new"])
    if c["kind"] == "attn":
        return tq.tq_kv_attention(h, 0, st["q"], cu_q=None if c["nq"] == 1 else st["cu"], max_q=c["nq"],
                                  max_len=c["maxlen"], window=c["window"], out_f32=c["f32"], want_lse=True)
    if c["kind"] == "fork":
        tq.tq_kv_free(h, st["children"])
        tq.tq_kv_fork(h, st["parents"], st["children"])
    else:
        for slots, cu in st["halves"]:
            tq.tq_kv_free(h, slots)
            tq.tq_kv_compact(h)
            tq.tq_kv_extend(h, cu_new=cu, seqs=slots)
    return st["pages"], st["lens"], st["refs"], st["data"]


def run(st):
    c = st["case"]
    if own:
        return _own(st, c)
    return {"q4": _plain_q4, "append": _plain_append, "attn": _plain_attn, "fork": _plain_fork,
            "churn": _plain_churn}[c["kind"]](st, c)


# --------------------------------------------------------------------------
# The definitions in 64 bits, element by element from where the layouts put
# each code.
# --------------------------------------------------------------------------

def _nib(buf, word, e_nibble):
    """Codes at nibble `e_nibble` of 32-bit word `word` of a byte buffer."""
    return ((buf[word * 4 + e_nibble // 2].long() >> (4 * (e_nibble % 2))) & 15).double()


def _exact_q4(c, st):
    n, k, g = c["n"], c["k"], c["g"]
    kb = -(-k // 128)
    nib = torch.tensor(NIBBLE, device="cuda")
    i = torch.arange(k, device="cuda")
    blk, j, cc, e = i // 128, i % 128 // 32, i % 32 // 8, i % 8
    x = st["x"].double()
    pairs = st["params"].double().view(-1, 2)
    y = torch.empty((c["b"], n), dtype=torch.float64, device="cuda")
    for r in range(0, n, 8192):
        row = torch.arange(r, min(n, r + 8192), device="cuda")[:, None]
        q = _nib(st["codes"], ((row // 16 * kb + blk) * 64 + cc * 16 + row % 16) * 4 + j, nib[e])
        at = (row // 16 * (kb * 128 // g) + i // g) * 16 + row % 16
        y[:, r:r + 8192] = x @ (q * pairs[at, 0] + pairs[at, 1]).t()
    return y


def _exact_rows(c, st, seq, pos, which):
    """float64 keys (which 0) or values (1) [H, T, D] of positions `pos`."""
    d, g, ps, H = c["d"], c["g"], c["ps"], c["hkv"]
    rec, nb = _rec(c), c["ps"] // 32
    page = st["pages"][seq].long()[pos // ps]
    t, i, h = pos % 32, torch.arange(d, device="cuda"), torch.arange(H, device="cuda")
    base = (page * H * nb + h[:, None] * nb + pos % ps // 32) * rec                      # [H, T]
    base, t = base[..., None], t[:, None]
    flat = st["data"][0].reshape(-1)
    if which == 0:
        word = ((t // 16 * 4 + i % 32 // 8) * 16 + t % 16) * (d // 32) + i // 32
        q = _nib(flat, base // 4 + word, torch.tensor(NIBBLE, device="cuda")[i % 8])
    else:
        word = ((i // 64 * 4 + t % 16 // 4) * 16 + i % 16) * 4 + i % 64 // 16
        q = _nib(flat, base // 4 + 4 * d + word, t // 16 * 4 + t % 4)
    at = (base + 32 * d + which * 128 * (d // g)) // 4 + i // g * 32 + t
    pairs = flat.view(torch.float16).double().view(-1, 2)
    return q * pairs[at, 0] + pairs[at, 1]


def _exact_attn(c, st):
    b, nq, hq, H, d = c["b"], c["nq"], c["hq"], c["hkv"], c["d"]
    out = torch.zeros((b * nq, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((b * nq, hq), -math.inf, dtype=torch.float64, device="cuda")
    for s, ln in enumerate(_lens(c)):
        if ln == 0:
            continue
        pos = torch.arange(ln, device="cuda")
        k, v = _exact_rows(c, st, s, pos, 0), _exact_rows(c, st, s, pos, 1)
        for h in range(hq):
            q = st["q"][s * nq:(s + 1) * nq, h].double()
            a = q @ k[h // (hq // H)].t() / math.sqrt(d)
            qp = ln - nq + torch.arange(nq, device="cuda")[:, None]
            hide = (pos > qp) | ((pos <= qp - c["window"]) if c["window"] else (pos < 0))
            a = a.masked_fill(hide, -math.inf)
            lse[s * nq:(s + 1) * nq, h] = torch.logsumexp(a, -1)
            out[s * nq:(s + 1) * nq, h] = torch.softmax(a, -1) @ v[h // (hq // H)]
    return out, lse


def _exact_append(c, st):
    outs = []
    for x in (st["k"], st["v"]):
        w = x.double().unflatten(-1, (-1, c["g"]))
        lo, hi = w.min(-1, keepdim=True).values, w.max(-1, keepdim=True).values
        s = ((hi - lo) / 15).half().double()
        q = torch.clamp(torch.round((w - lo) / s), 0, 15)
        outs.append((q * s + lo).flatten(-2))
    return tuple(outs)


def exact(c, seed):
    """What run() gives in 64 bits; the page operators give whole numbers
    only, which have no nearer value."""
    if c["kind"] in ("fork", "churn"):
        return None
    st = prepare(c, seed)
    return {"q4": _exact_q4, "attn": _exact_attn, "append": _exact_append}[c["kind"]](c, st)
