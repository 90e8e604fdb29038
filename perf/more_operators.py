"""Performance cases of what a decode step does between its projections and
its cache and behind its output head: rotary positions, attention with a
window and first tokens that stay visible, attention of rows that share a
prefix, and the log probabilities of the logits.

A case is one of four kinds of work:

* ``rope``    rotary positions of several axes on the queries and keys of a
              call, in one pass: ``tq_rope``;
* ``window``  attention over the 4-bit paged cache with a sliding window and
              the first tokens of every sequence beside it:
              ``tq_kv_attention(window=, sinks=)``;
* ``shared``  attention over the 4-bit paged cache of groups of rows whose
              first tokens lie in the same pages:
              ``tq_kv_attention(prefix=, groups=)``;
* ``logp``    log probabilities of given tokens, the entropy and the most
              likely tokens of rows of logits: ``tq_logprobs``.

``own`` chooses between the library's calls and the plain form: elementary
torch operations in 32 bits (angles in 64) on the same buffers.

The packed layout of the cache.  Eight 4-bit codes make a 32-bit word; element
e of the eight sits in nibble NIBBLE[e].  A page holds, per key/value head,
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

NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)      # element e of eight -> nibble of the word
ORDER = (0, 2, 4, 6, 1, 3, 5, 7)       # nibble -> element
HQ, HKV, D = 32, 8, 128                # heads of the decoder layer of the package's synthetic workloads
MOST_LOGITS = 75_000_000
MOST_ROTATED = 8191 * (HQ + HKV) * D


def listed():
    return [
        # The step of one user at a far position: latency.
        rope("rope 1 token", 1, start=900_001),
        # A long prompt of text, images and video: three axes, the channel pairs
        # dealt out in sections, q and k inside the output of one projection.
        rope("rope 8191 3 axes", 8191, axes=3, fused=True),
        # A serving batch of ragged lengths behind a window, an idle slot.
        window("window b32 to 8192", 32, 8192, window=1024, sinks=4),
        # One user with a long document and a wide window.
        window("window b1 len 131072", 1, 131072, window=16384, sinks=64, g=128),
        # Prompts in chunks, smaller heads; the last sink ends inside a tile;
        # fp32 outputs and their log-sum.
        window("window chunk 2x700 d64", 2, 5000, nq=700, hq=14, hkv=2, d=64, g=32, window=777, sinks=37, f32=True),
        # A few branches of a short prompt: latency.
        shared("shared 3 over 256", 3, 1, 256, 44, hq=8, hkv=2, ps=32),
        # Sixteen samples of one prompt.
        shared("shared 16 over 8000", 16, 1, 8000, 500),
        # Sixty-four users behind one long instruction.
        shared("shared 64 over 32768", 64, 1, 32768, 512),
        # Several prompts of different lengths, some rows each, three drafted
        # tokens a row, smaller heads, fp32 outputs and their log-sum.
        shared("shared 4x12 d64 g32", 12, 4, 4096, 200, nq=3, hq=14, hkv=2, d=64, g=32, f32=True),
        # The next token of one row over a small vocabulary, some alternatives.
        logp("logp 1x5000", 1, 5000, k=3),
        # A serving batch over a large vocabulary, logits as the head gives them.
        logp("logp 64x131072 f32", 64, 131072, k=20, f32=True),
        # A long text scored, a few given tokens a row, an odd vocabulary with
        # tokens ruled out, rows that lie further apart than they are long.
        logp("logp 1500x49999 masked", 1500, 49999, k=1, m=3, masked=True, pad=33),
    ]


def rope(name, t, axes=1, hq=HQ, hkv=HKV, d=D, rot=None, start=0, dealt=False, adjacent=False, inverse=False,
         fused=False, scale=1.0):
    return dict(name=name, kind="rope", t=t, axes=axes, hq=hq, hkv=hkv, d=d, rot=rot or d, start=start, dealt=dealt,
                adjacent=adjacent, inverse=inverse, fused=fused, scale=scale)


def window(name, b, maxlen, nq=1, hq=HQ, hkv=HKV, d=D, g=64, ps=64, window=1024, sinks=4, f32=False, mix=1):
    return dict(name=name, kind="window", b=b, maxlen=maxlen, nq=nq, hq=hq, hkv=hkv, d=d, g=g, ps=ps, window=window,
                sinks=sinks, f32=f32, mix=mix)


def shared(name, rows, groups, prefix, tail, nq=1, hq=HQ, hkv=HKV, d=D, g=64, ps=64, f32=False, mix=1):
    return dict(name=name, kind="shared", rows=rows, groups=groups, prefix=prefix, tail=tail, nq=nq, hq=hq, hkv=hkv,
                d=d, g=g, ps=ps, f32=f32, mix=mix)


def logp(name, t, v, k=0, m=1, f32=False, masked=False, pad=0, scale=1.0):
    return dict(name=name, kind="logp", t=t, v=v, k=k, m=m, f32=f32, masked=masked, pad=pad, scale=scale)


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["rope", "rope", "window", "window", "window", "shared", "shared", "shared", "shared", "logp",
                       "logp", "logp"])
    mix = rng.randrange(1, 1 << 20)
    d = rng.choice([64, 128, 128])
    g = rng.choice([v for v in (32, 64, 64, 128) if v <= d])
    ps = rng.choice([32, 64, 64, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    if kind == "rope":
        d = rng.choice([64, 96, 128, 128, 256])
        hq = hkv * rng.choice([1, 2, 4, 4, 7, 8])
        t = log_int(1, min(8191, MOST_ROTATED // (d * (hq + hkv))))
        rot = rng.choice([d, d, d, d // 2, d // 4])
        c = rope("", t, rng.choice([1, 1, 2, 3, 3]), hq, hkv, d, rot, rng.choice([0, log_int(1, 1_000_000)]),
                 rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.5,
                 rng.choice([1.0, 1.0, 1.25]))
    elif kind == "window":
        nq = rng.choice([1, 1, 1, log_int(2, 16), log_int(17, 700)])
        share = rng.choice([1, 2, 4, 4, 7, 8, 16] if nq <= 16 else [1, 2, 4])
        b = log_int(1, 64 if nq == 1 else 8 if nq <= 16 else 2)
        most = (131072 if nq == 1 else 16384 if nq <= 16 else 5000) // (b if nq == 1 else 1)
        c = window("", b, nq + log_int(30, most), nq, share * hkv, hkv, d, g, ps, log_int(16, 16384),
                   rng.choice([1, 4, log_int(1, 256)]), rng.random() < 0.3, mix)
    elif kind == "shared":
        nq = rng.choice([1, 1, 1, log_int(2, 8)])
        share = rng.choice([1, 2, 4, 4, 7, 8])
        groups = rng.choice([1, 1, 2, log_int(2, 6)])
        rows = log_int(2, 64 // groups)
        most = 64 * 32768 * HQ // (rows * groups * nq * share * hkv)
        prefix = -(-log_int(ps, max(ps, min(32768, most))) // ps) * ps
        c = shared("", rows, groups, prefix, nq + log_int(1, 500), nq, share * hkv, hkv, d, g, ps, rng.random() < 0.3,
                   mix)
    else:
        v = log_int(100, 131072)
        t = log_int(1, min(4096, max(1, MOST_LOGITS // v // 2)))
        c = logp("", t, v, rng.choice([0, 1, rng.randint(2, 32), rng.randint(2, 32)]), rng.randint(1, 4),
                 rng.random() < 0.5, rng.random() < 0.4, rng.choice([0, 0, rng.randint(1, 64)]),
                 rng.choice([1.0, 1.0, 1.25, 0.7]))
    c.pop("name", None)
    return c


# --------------------------------------------------------------------------
# Sizes of a case.
# --------------------------------------------------------------------------

def _spread(r, hi, lo):
    return max(lo, min(hi, round(math.exp(r.uniform(math.log(lo), math.log(max(lo, hi)))))))


def _groups(c):
    """Rows and shared tokens of every group: the first the largest, the others
    spread over their logarithm; what is shared fills its pages."""
    r = random.Random(c["mix"])
    ps = c["ps"]
    rows = [c["rows"]] + [_spread(r, c["rows"], 1) for _ in range(c["groups"] - 1)]
    return rows, [c["prefix"]] + [-(-_spread(r, c["prefix"], ps) // ps) * ps for _ in range(c["groups"] - 1)]


def _lens(c):
    """Tokens in the cache of every sequence, spread over their logarithm, the
    longest first; one idle slot (no tokens) in a batch of eight or more single
    tokens."""
    r = random.Random(c["mix"] + 1)
    if c["kind"] == "shared":
        rows, prefix = _groups(c)
        v = [p + _spread(r, c["tail"], c["nq"]) for n, p in zip(rows, prefix) for _ in range(n)]
        v[0] = prefix[0] + c["tail"]
        return v
    hi, lo = c["maxlen"], max(c["nq"], c["maxlen"] // 16, 1)
    v = [hi] + [_spread(r, hi, lo) for _ in range(c["b"] - 1)]
    if c["nq"] == 1 and c["b"] >= 8:
        v[3] = 0
    return v


def _rec(c):
    """Bytes of one record: 32 tokens of one head, keys and values."""
    return 32 * (c["d"] + 8 * c["d"] // c["g"])


def _pages(n, ps):
    return -(-n // ps)


def _seen(pos, w, sinks):
    """Tokens that a query at `pos` attends to."""
    first = max(0, pos + 1 - w)
    return pos + 1 - first + min(sinks, first)


def work(c):
    if c["kind"] == "rope":
        n = c["t"] * (c["hq"] + c["hkv"])
        return {"bytes": 4 * n * c["d"] + 4 * c["axes"] * c["t"] + 3 * c["rot"], "flops": 3 * n * c["rot"]}
    if c["kind"] == "logp":
        n = c["t"] * c["v"]
        return {"bytes": n * (4 if c["f32"] else 2) + c["t"] * (4 + 8 * (c["k"] + c["m"])), "flops": 6 * n}
    per = c["hkv"] * (c["d"] + 8 * c["d"] // c["g"])               # bytes of a token, keys and values
    lens = _lens(c)
    rows = len(lens) * c["nq"] * c["hq"]
    if c["kind"] == "shared":
        read = sum(lens) - sum((n - 1) * p for n, p in zip(*_groups(c)))
        pairs = sum(c["nq"] * ln - c["nq"] * (c["nq"] - 1) // 2 for ln in lens)
    else:
        w, s, nq = c["window"], c["sinks"], c["nq"]
        read = sum(min(ln, w + nq - 1) + min(s, max(0, ln - nq + 1 - w)) for ln in lens)
        pairs = sum(_seen(p, w, s) for ln in lens for p in range(max(0, ln - nq), ln))
    return {"bytes": read * per + rows * c["d"] * (2 + (4 if c["f32"] else 2)) + rows * 4,
            "flops": 4 * pairs * c["hq"] * c["d"]}


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
    """Codes (uint8, as x) and (scale, offset) fp16 [..., last/g, 2] of fp16 x."""
    xg = x.float().unflatten(-1, (-1, g))
    lo = xg.amin(-1, keepdim=True)
    s = ((xg.amax(-1, keepdim=True) - lo) / 15.0).half()
    sf = s.float()
    q = torch.where(sf > 0, torch.round((xg - lo) / sf).clamp(0, 15), torch.zeros_like(xg)).to(torch.uint8)
    return q.flatten(-2), torch.cat([s, lo.half()], -1)


def _nibbles(q):
    """uint8 codes [..., 8] (in nibble order) -> bytes [..., 4]."""
    return q[..., 0::2] | (q[..., 1::2] << 4)


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


def _table(c, seed, lens):
    """Page table [n_seqs, max_pages], lengths and counts for sequences of
    these lengths, their pages in random order over a pool with a few spare
    ones; rows of a group name the same pages for what they share."""
    ps = c["ps"]
    common = [0] * len(lens)                                    # pages that a row takes over from the row `lead`
    lead = list(range(len(lens)))
    if c["kind"] == "shared":
        at = 0
        for n, p in zip(*_groups(c)):
            for r in range(at + 1, at + n):
                common[r], lead[r] = p // ps, at
            at += n
    need = [_pages(ln, ps) for ln in lens]
    total = sum(need) - sum(common) + len(lens) + 5
    order = torch.randperm(total, generator=_gen(seed, 7), device="cuda").to(torch.int32).cpu()
    pages = torch.full((len(lens), max(need + [1]) + 1), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        pages[s, :common[s]] = pages[lead[s], :common[s]]
        pages[s, common[s]:n] = order[at:at + n - common[s]]
        at += n - common[s]
    refs = torch.bincount(pages[pages >= 0].long(), minlength=total).to(torch.int32)
    return pages.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), refs.cuda(), total


def _pool(c, seed, total):
    out = []
    for at in range(0, total, 4096):                            # fp16 copies of a large pool are not kept
        shape = (min(4096, total - at), c["hkv"], c["ps"], c["d"])
        g = _gen(seed, 11, at)
        out.append(_pack_pages(_rows(shape, g), _rows(shape, g), c["g"]))
    return torch.cat(out)[None]


def _positions(c, seed):
    """One axis: a text from `start` on.  Several: texts between pictures, whose
    tokens lie on a grid (time, height, width) that starts where the text ended."""
    t, axes, start = c["t"], c["axes"], c["start"]
    if axes == 1:
        return torch.arange(start, start + t, device="cuda", dtype=torch.int32)
    r = random.Random(seed)
    parts, n, at = [], 0, start
    while n < t:
        text = torch.arange(at, at + r.randint(1, 60)).expand(axes, -1)
        at += text.shape[1]
        f, h, w = r.randint(1, 4), r.randint(1, 24), r.randint(1, 24)
        grid = torch.stack([x.flatten() for x in torch.meshgrid(torch.arange(f), torch.arange(h), torch.arange(w),
                                                                indexing="ij")])[-axes:] + at
        at += max(f, h, w)
        parts += [text, grid]
        n += text.shape[1] + grid.shape[1]
    return torch.cat(parts, 1)[:, :t].to(torch.int32).cuda()


def prepare(c, seed):
    st = {"case": dict(c)}
    g = _gen(seed, 1)
    if c["kind"] == "rope":
        t, hq, hkv, d, n = c["t"], c["hq"], c["hkv"], c["d"], c["rot"] // 2
        if c["fused"]:                                          # [q | k | v] of one projection
            x = _rows((t, hq + 2 * hkv, d), g)
            st["q"], st["k"] = x[:, :hq], x[:, hq:hq + hkv]
        else:
            st["q"], st["k"] = _rows((t, hq, d), g), _rows((t, hkv, d), g)
        st["pos"] = _positions(c, seed)
        st["freq"] = (10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n)).float()
        if c["axes"] > 1:
            i = torch.arange(n, device="cuda")
            st["axis"] = (i % c["axes"] if c["dealt"] else i * c["axes"] // n).to(torch.uint8)
        return st
    if c["kind"] == "logp":
        t, v = c["t"], c["v"]
        dtype = torch.float32 if c["f32"] else torch.float16
        x = torch.empty((t, v + c["pad"]), dtype=dtype, device="cuda")[:, :v]
        for at in range(0, t, 256):                             # a few likely tokens over a broad floor
            z = torch.randn((min(256, t - at), v), generator=g, device="cuda")
            u = torch.rand((z.shape[0], v), generator=g, device="cuda")
            z = 2.0 * z - 4.0 + torch.where(u < 20.0 / v, 12.0 * torch.rand(z.shape, generator=g, device="cuda"), 0.0)
            if c["masked"]:
                z = z.masked_fill(torch.rand((z.shape[0], v), generator=g, device="cuda") < 0.3, -math.inf)
            x[at:at + 256] = z.to(dtype)
        st["x"] = x
        st["ids"] = torch.randint(0, v, (t, c["m"]), generator=g, device="cuda", dtype=torch.int32)
        st["ids"][:, 0] = x.float().argmax(-1).int()            # mostly what was sampled is likely
        return st
    lens = _lens(c)
    b = len(lens)
    pages, lens_t, refs, total = _table(c, seed, lens)
    st.update(pages=pages, lens=lens_t, refs=refs, data=_pool(c, seed, total))
    st["q"] = torch.randn((b * c["nq"], c["hq"], c["d"]), generator=g, device="cuda", dtype=torch.float16)
    st["cu"] = torch.arange(0, b * c["nq"] + 1, c["nq"], device="cuda", dtype=torch.int32)
    if c["kind"] == "shared":
        rows, prefix = _groups(c)
        st["prefix"] = torch.tensor([p for r, p in zip(rows, prefix) for _ in range(r)], dtype=torch.int32).cuda()
        st["shared"] = torch.tensor(prefix).cuda()
        st["groups"] = torch.tensor([0] + torch.tensor(rows).cumsum(0).tolist(), dtype=torch.int32).cuda()
        # row of the call -> group and place in it; the other way round, filled up with row 0
        n, m = c["groups"], max(rows)
        st["group_of"] = torch.tensor([i for i, r in enumerate(rows) for _ in range(r)]).cuda()
        st["place_of"] = torch.tensor([k for r in rows for k in range(r)]).cuda()
        st["row_at"] = torch.zeros((n, m), dtype=torch.int64, device="cuda")
        st["row_at"][st["group_of"], st["place_of"]] = torch.arange(b, device="cuda")
    return st


# --------------------------------------------------------------------------
# The plain form: the definitions in 32 bits, on the packed bytes.
# --------------------------------------------------------------------------

def _plain_rope(st, c):
    n, d = c["rot"] // 2, c["d"]
    pos = st["pos"].double() if c["axes"] == 1 else st["pos"].double()[st["axis"].long()].t()     # [T] or [T, n]
    a = (pos[:, None] if c["axes"] == 1 else pos) * st["freq"].double()
    cos, sin = (c["scale"] * torch.cos(a)).float()[:, None], (c["scale"] * torch.sin(a)).float()[:, None]
    if c["inverse"]:
        sin = -sin
    out = []
    for x in (st["q"], st["k"]):
        y = x.float()
        r = y[..., :c["rot"]]
        x1, x2 = (r[..., 0::2], r[..., 1::2]) if c["adjacent"] else (r[..., :n], r[..., n:])
        parts = [x1 * cos - x2 * sin, x2 * cos + x1 * sin]
        r = torch.stack(parts, -1).flatten(-2) if c["adjacent"] else torch.cat(parts, -1)
        out.append((torch.cat([r, y[..., c["rot"]:]], -1) if c["rot"] < d else r).half())
    return tuple(out)


def _plain_logp(st, c):
    raw = st["x"].float()
    x = raw * c["scale"]
    top = x.amax(-1, keepdim=True)
    below = x - top
    e = torch.exp(below)
    s = e.sum(-1, keepdim=True)
    log_s = torch.log(s)
    entropy = (log_s - torch.where(e > 0, e * below, 0.0).sum(-1, keepdim=True) / s)[:, 0]
    logp = x.gather(1, st["ids"].long()) - top - log_s
    if c["k"] == 0:
        return logp, entropy
    # The larger logit first, of equal ones the lower index: one whole number each.
    bits = (raw + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) - torch.arange(c["v"], device="cuda")
    ids = (-torch.topk(order, c["k"], -1).values) & 0xFFFFFFFF
    return logp, entropy, ids.int(), x.gather(1, ids) - top - log_s


def _codes(b):
    """bytes [..., 4] -> codes [..., 8] in element order."""
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)[..., list(NIBBLE)]


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

    def values(q, at):
        p = raw[..., at:at + 128 * d // g].contiguous().view(torch.float16).view(P, H, nb, d // g, 32, 2)
        p = p.permute(0, 1, 2, 4, 3, 5).reshape(P, H, nb * 32, d // g, 2).float()
        return (q.float() * p[..., :1] + p[..., 1:]).flatten(-2)

    return values(qk, 32 * d), values(qv, 32 * d + 128 * d // g)


def _plain_rows(st, c, pages):
    """fp32 keys and values [rows, H, n ps, D] of page numbers [rows, n]."""
    n, m = pages.shape
    k, v = _plain_pages(st["data"][0][pages.clamp(min=0).reshape(-1)], c)
    return tuple(x.view(n, m, c["hkv"], c["ps"], c["d"]).transpose(1, 2).reshape(n, c["hkv"], m * c["ps"], c["d"])
                 for x in (k, v))


def _plain_sums(q, k, v, see):
    """Largest logit, sum of exponentials and weighted values of queries q
    [n, H, R, D] over keys and values [n, H, T, D] that they see [n, 1, R, T]."""
    s = (q @ k.transpose(2, 3).contiguous()) * (q.shape[-1] ** -0.5)
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - top.clamp(min=-1e30))
    return top, e.sum(-1, keepdim=True), e @ v


def _plain_out(c, top, l, o, b):
    """o and lse by token and head from [b, H, share * nq, ...]."""
    o = o / torch.where(l > 0, l, 1.0)
    lse = (top + torch.log(l))[..., 0]
    nq, share = c["nq"], c["hq"] // c["hkv"]
    o = o.view(b, c["hkv"], share, nq, c["d"]).permute(0, 3, 1, 2, 4).reshape(b * nq, c["hq"], c["d"])
    lse = lse.view(b, c["hkv"], share, nq).permute(0, 3, 1, 2).reshape(b * nq, c["hq"]).contiguous()
    return (o if c["f32"] else o.half()), lse


def _plain_queries(st, c, b):
    """fp32 queries [b, H, share * nq, D]."""
    share = c["hq"] // c["hkv"]
    q = st["q"].float().view(b, c["nq"], c["hkv"], share, c["d"]).permute(0, 2, 3, 1, 4)
    return q.reshape(b, c["hkv"], share * c["nq"], c["d"])


def _plain_window(st, c):
    b, nq, ps, w = c["b"], c["nq"], c["ps"], c["window"]
    share, mp = c["hq"] // c["hkv"], st["pages"].shape[1]
    lens = st["lens"].long()[:, None]
    # The pages of the sinks, then those of the windows.
    front = min(mp, _pages(c["sinks"], ps))
    first = (lens - nq + 1 - w).clamp(min=0) // ps
    col = torch.cat([torch.arange(front, device="cuda").expand(b, -1),
                     first + torch.arange(min(mp, _pages(w + nq, ps) + 1), device="cuda")], 1)       # [b, n]
    pages = st["pages"].long().gather(1, col.clamp(max=mp - 1))
    k, v = _plain_rows(st, c, pages)
    j = (col[..., None] * ps + torch.arange(ps, device="cuda")).flatten(1)                         # [b, T]
    twice = torch.arange(j.shape[1], device="cuda") >= front * ps
    there = (j < lens) & ~(twice & (j < front * ps))
    pos = (lens - nq + torch.arange(nq, device="cuda"))[..., None]                                 # [b, nq, 1]
    see = there[:, None] & (j[:, None] <= pos) & ((j[:, None] > pos - w) | (j[:, None] < c["sinks"]))
    v = v.masked_fill(~there[:, None, :, None], 0.0)
    return _plain_out(c, *_plain_sums(_plain_queries(st, c, b), k, v, see.repeat(1, share, 1)[:, None]), b)


def _plain_shared(st, c):
    ps, nq, H, d = c["ps"], c["nq"], c["hkv"], c["d"]
    share, b = c["hq"] // H, st["lens"].numel()
    n, m = st["row_at"].shape
    q = _plain_queries(st, c, b)
    prefix = st["shared"]
    # What a group shares, once: the queries of all its rows beside each other.
    k, v = _plain_rows(st, c, st["pages"].long()[st["row_at"][:, 0], :c["prefix"] // ps])
    j = torch.arange(c["prefix"], device="cuda")
    v = v.masked_fill(~(j < prefix[:, None])[:, None, :, None], 0.0)
    qs = q[st["row_at"]].transpose(1, 2).reshape(n, H, m * share * nq, d)
    part = _plain_sums(qs, k, v, (j < prefix[:, None])[:, None, None])
    top1, l1, o1 = (x.view(n, H, m, share * nq, -1).transpose(1, 2)[st["group_of"], st["place_of"]] for x in part)
    # What every row has behind it.
    first, lens = st["prefix"].long()[:, None], st["lens"].long()[:, None]
    col = first // ps + torch.arange(_pages(c["tail"], ps), device="cuda")
    k, v = _plain_rows(st, c, st["pages"].long().gather(1, col.clamp(max=st["pages"].shape[1] - 1)))
    j = first + torch.arange(k.shape[2], device="cuda")
    v = v.masked_fill(~(j < lens)[:, None, :, None], 0.0)
    pos = (lens - nq + torch.arange(nq, device="cuda"))[..., None]
    see = (j[:, None] <= pos).repeat(1, share, 1)[:, None]
    top2, l2, o2 = _plain_sums(q, k, v, see)
    top = torch.maximum(top1, top2)
    w1, w2 = torch.exp(top1 - top), torch.exp(top2 - top)
    return _plain_out(c, top, l1 * w1 + l2 * w2, o1 * w1 + o2 * w2, b)


# --------------------------------------------------------------------------
# The library's calls.
# --------------------------------------------------------------------------

def _own(st, c):
    from paper_2609_09240_amd import tq
    if c["kind"] == "rope":
        return tq.tq_rope(st["q"], st["k"], st["pos"], st["freq"], axis=st.get("axis"), adjacent=c["adjacent"],
                          inverse=c["inverse"], scale=c["scale"])
    if c["kind"] == "logp":
        logp, entropy, ids, top = tq.tq_logprobs(st["x"], st["ids"], top=c["k"], scale=c["scale"], want_entropy=True)
        return (logp, entropy, ids, top) if c["k"] else (logp, entropy)
    if "handle" not in st:                                      # made once and kept beside its buffers
        st["handle"] = tq.KVCache(st["data"], st["pages"], st["lens"], st["refs"], n_kv_heads=c["hkv"],
                                  head_dim=c["d"], page_size=c["ps"], group=c["g"])
    cu = None if c["nq"] == 1 else st["cu"]
    if c["kind"] == "window":
        return tq.tq_kv_attention(st["handle"], 0, st["q"], cu_q=cu, max_q=c["nq"], max_len=c["maxlen"],
                                  window=c["window"], sinks=c["sinks"], out_f32=c["f32"], want_lse=True)
    return tq.tq_kv_attention(st["handle"], 0, st["q"], cu_q=cu, max_q=c["nq"], max_len=c["prefix"] + c["tail"],
                              prefix=st["prefix"], groups=st["groups"], max_prefix=c["prefix"], max_tail=c["tail"],
                              out_f32=c["f32"], want_lse=True)


def run(st):
    c = st["case"]
    if own:
        return _own(st, c)
    return {"rope": _plain_rope, "logp": _plain_logp, "window": _plain_window, "shared": _plain_shared}[c["kind"]](st, c)


# --------------------------------------------------------------------------
# The definitions in 64 bits, element by element.
# --------------------------------------------------------------------------

def _exact_rope(c, st):
    n, out = c["rot"] // 2, []
    pos = st["pos"].view(c["axes"], c["t"]).double()
    axis = st["axis"].long() if "axis" in st else torch.zeros(n, dtype=torch.int64, device="cuda")
    for x in (st["q"], st["k"]):
        y = x.double().clone()
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + n)
            z = torch.complex(x[..., a].double(), x[..., b].double())
            angle = pos[axis[i]] * st["freq"][i].double() * (-1.0 if c["inverse"] else 1.0)
            z = z * torch.polar(torch.full_like(angle, c["scale"]), angle)[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_logp(c, st):
    logp = torch.empty((c["t"], c["m"]), dtype=torch.float64, device="cuda")
    entropy = torch.empty(c["t"], dtype=torch.float64, device="cuda")
    best = torch.empty((c["t"], c["k"]), dtype=torch.float64, device="cuda")
    for at in range(0, c["t"], 128):
        s = slice(at, at + 128)
        z = st["x"][s].double() * c["scale"]
        lp = z - torch.logsumexp(z, -1, keepdim=True)
        logp[s] = lp.gather(1, st["ids"][s].long())
        entropy[s] = torch.special.entr(torch.exp(lp)).sum(-1)
        best[s] = torch.sort(lp, -1, descending=True).values[:, :c["k"]]
    return (logp, entropy, None, best) if c["k"] else (logp, entropy)


def _nib(buf, word, e_nibble):
    """Codes at nibble `e_nibble` of 32-bit word `word` of a byte buffer."""
    return ((buf[word * 4 + e_nibble // 2].long() >> (4 * (e_nibble % 2))) & 15).double()


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
    nq, hq, H, d = c["nq"], c["hq"], c["hkv"], c["d"]
    lens = _lens(c)
    out = torch.zeros((len(lens) * nq, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((len(lens) * nq, hq), -math.inf, dtype=torch.float64, device="cuda")
    for s, ln in enumerate(lens):
        if ln == 0:
            continue
        pos = torch.arange(ln, device="cuda")
        qp = ln - nq + torch.arange(nq, device="cuda")[:, None]
        hide = pos > qp
        if c["kind"] == "window":
            hide |= (pos <= qp - c["window"]) & (pos >= c["sinks"])
        k, v = _exact_rows(c, st, s, pos, 0), _exact_rows(c, st, s, pos, 1)
        for h in range(hq):
            q = st["q"][s * nq:(s + 1) * nq, h].double()
            a = (q @ k[h // (hq // H)].t() / math.sqrt(d)).masked_fill(hide, -math.inf)
            lse[s * nq:(s + 1) * nq, h] = torch.logsumexp(a, -1)
            out[s * nq:(s + 1) * nq, h] = torch.softmax(a, -1) @ v[h // (hq // H)]
    return out, lse


def exact(c, seed):
    """What run() gives in 64 bits."""
    st = prepare(c, seed)
    return {"rope": _exact_rope, "logp": _exact_logp}.get(c["kind"], _exact_attn)(c, st)
