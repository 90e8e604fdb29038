"""Plain CPU reference (numpy, fp64) of what a decode step does around its
projections, its cache and its output head: rotary positions, attention with
sinks beside a window, the tokens that rows share, log probabilities."""

import numpy as np


def rope(x, positions, freq, axis=None, adjacent=False, inverse=False, scale=1.0):
    """x [T, heads, D] with its first 2 n channels turned, n = len(freq):
    positions [T] or [axes, T], axis [n] (axis 0 without; a pair of an axis that is
    not there is not turned)."""
    y = np.array(x, dtype=np.float64)
    pos = np.atleast_2d(np.asarray(positions, dtype=np.float64))
    n = len(freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
        ax = 0 if axis is None else int(axis[i])
        angle = (pos[ax] if ax < pos.shape[0] else 0 * pos[0]) * np.float64(freq[i])
        if inverse:
            angle = -angle
        c, s = scale * np.cos(angle)[:, None], scale * np.sin(angle)[:, None]
        x1, x2 = np.asarray(x[..., a], np.float64), np.asarray(x[..., b], np.float64)
        y[..., a], y[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def attention(q, k, v, scale, window=0, sinks=0):
    """As oracle.q4.attention, with the first `sinks` tokens beside the window."""
    n, L = q.shape[0], k.shape[0]
    o, lse, p = np.zeros((n, k.shape[1])), np.full(n, -np.inf), np.zeros((n, L))
    j = np.arange(L)
    for i in range(n):
        pos = L - n + i
        see = j <= pos
        if window:
            see &= (j > pos - window) | (j < sinks)
        if not see.any():
            continue
        a = scale * (k[see].astype(np.float64) @ q[i].astype(np.float64))
        top = a.max()
        e = np.exp(a - top)
        p[i, see] = e / e.sum()
        lse[i] = top + np.log(e.sum())
        o[i] = p[i, see] @ v[see].astype(np.float64)
    return o, lse, p


def shared_prefix(table, lens, page_size, n_pages, seqs, groups):
    """Tokens of every row in the leading pages that its group's rows name
    alike; rows that hold none, are alone or have no group: 0."""
    out = [0] * len(seqs)
    for g in range(len(groups) - 1):
        rows = [r for r in range(groups[g], groups[g + 1])
                if 0 <= seqs[r] < len(lens) and lens[seqs[r]] > 0]
        if len(rows) < 2:
            continue
        least = min(min(lens[seqs[r]], len(table[seqs[r]]) * page_size) for r in rows)
        pages = 0
        while pages * page_size < least:
            named = {table[seqs[r]][pages] for r in rows}
            if len(named) > 1 or not 0 <= min(named) < n_pages:
                break
            pages += 1
        for r in rows:
            out[r] = min(pages * page_size, least)
    return out


def logprobs(x, ids=None, top=0, scale=1.0):
    """(logp like ids, entropy [T], top ids [T, top], their logp) of logits x."""
    x = np.asarray(x, dtype=np.float64)
    T, V = x.shape
    ids = np.zeros((T, 0), np.int64) if ids is None else np.asarray(ids).reshape(T, -1)
    logp, ent = np.full(ids.shape, np.nan), np.full(T, np.nan)
    tops, tlp = np.zeros((T, top), np.int64), np.full((T, top), np.nan)
    for t in range(T):
        z = x[t] * scale
        order = np.lexsort((np.arange(V), -np.where(np.isnan(z), -np.inf, z)))
        tops[t] = order[:top]
        if np.isnan(z).any() or np.isposinf(z).any():
            continue
        m = z.max()
        if np.isneginf(m):
            lp, ent[t] = np.full(V, -np.inf), 0.0
        else:
            lp = z - m - np.log(np.exp(z - m).sum())
            p = np.exp(lp)
            ent[t] = -(p[p > 0] * lp[p > 0]).sum()
        for i, j in enumerate(ids[t]):
            if 0 <= j < V:
                logp[t, i] = lp[j]
        tlp[t] = lp[tops[t]]
    return logp, ent, tops, tlp
