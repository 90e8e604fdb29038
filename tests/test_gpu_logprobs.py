"""Log probabilities, entropies and most likely tokens against the fp64 oracle
(GPU).

Tolerance, with u = 2^-24, z = scale (x - max) <= 0, E = sum p |z|, E2 = sum p z^2.
An exponential is off by 2 u |z| (its argument: the constant, a product), 4 u of
its own and 2 u for each rescaling; the sums of a thread add at most V/256 + 64
terms (16 a chunk, and what is joined).  So log S is off by at most
    s = (2 E + 12 + V/256 + 64) u + 2 u log S,
a log probability by s + 4 u (|z| + |logp|), the entropy by
    s + (2 E2 + (12 + V/256 + 64) E) u + s E + 4 u (H + E).
(E = H - log S <= H.)
"""

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def logits(T, V, seed, f32, masked=0.0, spread=3.0):
    r = np.random.default_rng(seed)
    x = (spread * r.standard_normal((T, V))).astype(np.float32)
    x[r.random((T, V)) < masked] = -np.inf
    return x if f32 else x.astype(np.float16)


def check(x, got, ids=None, top=0, scale=1.0):
    logp, ent, tops, tlp = (None if t is None else t.cpu().numpy() for t in got)
    wl, we, wt, wtl = decode.logprobs(x, ids, top, scale)
    z = x.astype(np.float64) * scale
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = z.max(-1, keepdims=True)
        d = np.where(np.isfinite(z), m - z, 0.0)
        p = np.where(np.isfinite(z), np.exp(z - m), 0.0)
        S = p.sum(-1)
        S = np.where(S > 0, S, 1.0)                         # nothing possible: no term, nothing off
        E, E2, logS = (p * d).sum(-1) / S, (p * d * d).sum(-1) / S, np.log(S)
    n = x.shape[1] / 256 + 76
    s = (2 * E + n) * U + 2 * U * logS

    def near(a, w, bound, what):
        a = a.astype(np.float64)
        fine = np.isfinite(w)
        assert (np.isnan(a) == np.isnan(w)).all() and (a[~fine & ~np.isnan(w)] == w[~fine & ~np.isnan(w)]).all(), what
        err = np.abs(np.where(fine, a, 0.0) - np.where(fine, w, 0.0))
        assert (err[fine] <= np.broadcast_to(bound, w.shape)[fine]).all(), (what, float(np.nanmax(err)))

    if ids is not None:
        ids = np.asarray(ids).reshape(x.shape[0], -1)
        at = np.take_along_axis(d, np.clip(ids, 0, x.shape[1] - 1), 1)
        near(logp.reshape(ids.shape), wl, s[:, None] + 4 * U * (at + np.abs(np.where(np.isfinite(wl), wl, 0))), "logp")
    if ent is not None:
        near(ent, we, s + (2 * E2 + n * E) * U + s * E + 4 * U * (we + E), "entropy")
    if top:
        np.testing.assert_array_equal(tops, wt)
        at = np.take_along_axis(d, wt, 1)
        near(tlp, wtl, s[:, None] + 4 * U * (at + np.abs(np.where(np.isfinite(wtl), wtl, 0))), "top")


def run(x, ids=None, **kw):
    return tq.tq_logprobs(torch.from_numpy(x).cuda(), None if ids is None else torch.from_numpy(np.asarray(ids, np.int32)).cuda(),
                          want_entropy=True, **kw)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 2), (2, 31), (1, 257), (5, 1000), (2, 4095), (2, 4096), (3, 4097), (1, 8193),
                                 (2, 49999), (1, 131072), (3, 200001), (2500, 300), (70, 20000)])
def test_sizes(f32, T, V):
    r = np.random.default_rng(T + V)
    x = logits(T, V, V, f32)
    for top in sorted({0, 1, min(5, V), min(32, V)}):
        ids = r.integers(0, V, (T, 3))
        check(x, run(x, ids, top=top), ids, top)


@pytest.mark.parametrize("T,V", [(40, 4096), (3, 9000), (2, 131072)])
def test_every_number_of_tokens(T, V):
    x = logits(T, V, 13, V != 9000)
    order = decode.logprobs(x, None, 32)[2]
    for top in range(1, 33):
        np.testing.assert_array_equal(run(x, top=top)[2].cpu().numpy(), order[:, :top])


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("scale", [1.0, 0.3, 7.5])
def test_masks_ties_and_scales(f32, scale):
    """Ruled-out tokens, few that are left, values that come often."""
    for seed, masked in ((1, 0.3), (2, 0.999), (3, 0.9999)):
        x = logits(6, 30000, seed, f32, masked)
        x[3] = np.round(x[3])                               # ties everywhere
        x[4] = 0.25
        x[5] = -np.inf
        x[5, 17] = -3.0
        ids = np.stack([np.arange(6) * 5000, np.full(6, 17)], 1)
        check(x, run(x, ids, top=32, scale=scale), ids, 32, scale)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("scale", [1e-6, 333.0, 1e5, 1e9, 1e18])
def test_small_and_large_scales(f32, scale):
    """A small or a large temperature, up to one that leaves the largest logits alone."""
    x = logits(5, 9000, 8, f32, 0.1)
    x[1] += 100
    x[2] *= 1e-3
    x[3, 77] = x[3, 8888] = 60000                           # two of them, alike
    x[4] = -np.abs(x[4]) - 5000
    ids = np.tile([[77, 8888, 5]], (5, 1))
    check(x, run(x, ids, top=9, scale=scale), ids, 9, scale)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("V", [2, 300, 5000, 49999, 131072])
def test_a_token_that_is_nearly_certain(f32, V):
    """Of the others' sum, exponentials (2 |z| + 4), the sums of a thread, of lanes,
    waves and parts (V/256 + 64 + 12) and the logarithm (4) are off by u each; up to 16
    terms are added to -1 before the token's own 1, in steps of u / 2."""
    x = logits(6, V, 9, f32, 0.0, 1.0)
    at = np.array([0, V - 1, V // 2, V // 3, 1, V // 7])
    lead = np.log(V) + np.array([2.0, 4.0, 6.0, 9.0, 12.0, 15.0])
    x[np.arange(6), at] = x.max(-1) + lead
    got = run(x, at[:, None], top=1)
    check(x, got, at[:, None], 1)
    want = decode.logprobs(x, at[:, None], 1)[0][:, 0]
    z = (x.max(-1) - x.min(-1)).astype(np.float64)
    assert (want > -0.3).all() and (want < 0).all()
    for lp in (got[0][:, 0], got[3][:, 0]):
        assert (np.abs(lp.cpu().numpy() - want) <= (8 - want * (2 * z + 84 + V / 256)) * U).all()


def certain(T, V, f32, lead, at, rest):
    """Rows of `rest` with the largest logit at `at` and `lead` below it one at every
    place of V in turn; and those places."""
    places = [j for j in (0, 1, 3, 4, 7, 8, 9, 100, 255, 256, 1023, 1024, 2047, 2048, 2049, 4095, 4096, 4101, 12289, V // 2,
                          V - 9, V - 2, V - 1) if 0 <= j < V and j != at]
    x = np.full((len(places), V), rest, np.float32)
    x[:, at] = 20.0
    x[np.arange(len(places)), places] = 20.0 - lead
    return (x if f32 else x.astype(np.float16)), places


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("V", [2, 9, 300, 5000, 49999, 131072])
@pytest.mark.parametrize("rest", [-np.inf, -60.0])
def test_the_others_of_a_certain_token(f32, V, rest):
    """What is left of 1 is the others' sum, wherever they lie beside the certain token: in
    its thread, before and behind it, in other lanes, waves, chunks and parts.

    Relative to it alone, with u = 2^-24 and z up to 80: an argument of an exponential
    is off by 3 u z (constant, difference, product), the exponential by 4 u and 2 u for
    each of up to 8 rescalings, the sums by V/256 + 64 + 12 terms' u, the logarithm by 4
    u; the entropy's second sum by 4 u more, for its factors."""
    tol = (3 * 80 + 4 + 16 + V / 256 + 76 + 4 + 4) * U
    for at in sorted({0, 1, 5, 15, 77, 2050, 4097, V // 3, V - 1}):
        if at >= V:
            continue
        for lead in (2.0, 12.0, 18.5, 40.0, 79.0):
            x, places = certain(1, V, f32, lead, at, rest)
            if not places:
                continue
            ids = np.stack([np.full(len(places), at), places], 1)
            logp, ent, tops, tlp = (t.cpu().numpy().astype(np.float64) for t in run(x, ids, top=2))
            z = x.astype(np.float64) - 20.0
            p = np.exp(z)
            p[:, at] = 0.0
            others = p.sum(-1)
            log_s = np.log1p(others)
            want = log_s + (p * np.where(p > 0, -z, 0)).sum(-1) / (1 + others)
            assert (tops[:, 0] == at).all() and (logp[:, 0] == tlp[:, 0]).all()
            assert (np.abs(logp[:, 0] + log_s) <= tol * log_s).all(), (at, lead)
            assert (np.abs(ent - want) <= tol * want).all(), (at, lead)
            assert (np.abs(logp[:, 1] + lead + log_s) <= tol * (lead + log_s)).all(), (at, lead)


@pytest.mark.parametrize("f32", [False, True])
def test_certain_tokens_one_after_the_other(f32):
    """Every chunk's largest logit above the last one's, and what the old ones are then."""
    V = 45000
    for step in (3.0, 9.0, 17.5):
        x = np.full((9, V), -np.inf, np.float32)
        for i, at in enumerate(range(5, V, 4096)):
            for r in range(9):
                x[r, at + 3 * r] = i * step
                x[r, at + (r * 517) % 4000 + 40] = i * step - 8.0
        x = x if f32 else x.astype(np.float16)
        z = np.sort(x.astype(np.float64), -1)[:, ::-1] - x.max(-1, keepdims=True)
        others = np.exp(z[:, 1:]).sum(-1)
        want = np.log1p(others)
        got = tq.tq_logprobs(torch.from_numpy(x).cuda(), top=1)[3][:, 0].cpu().numpy().astype(np.float64)
        # as above, with z up to 183; what lies past 87 below, and is lost, is less than 2^-24 of it
        assert (np.abs(got + want) <= (3 * 183 + 105 + V / 256) * U * want).all(), step


@pytest.mark.parametrize("f32", [False, True])
def test_infinities_and_nan_beside_a_certain_token(f32):
    x = np.full((8, 9000), -40.0, np.float32)
    x[:, 4] = 30.0
    x[0, 3], x[1, 5], x[2, 5000], x[3, 0] = np.nan, np.nan, np.nan, np.inf
    x[4, 4], x[5, 8999] = np.inf, np.inf
    x[6, [3, 5]] = 30.0                                     # three alike
    x[7, 8999] = 30.0
    x = x if f32 else x.astype(np.float16)
    got = run(x, np.tile([[4, 8999]], (8, 1)), top=3)
    check(x, got, np.tile([[4, 8999]], (8, 1)), 3)


@pytest.mark.parametrize("f32", [False, True])
def test_nothing_possible_and_special_values(f32):
    x = logits(9, 9000, 4, f32)
    low = np.finfo(x.dtype).min
    x[0] = -np.inf
    x[1, 5000] = np.nan
    x[2, 7] = np.inf
    x[3] = low                                              # masks of the type's lowest value: all alike
    x[4, 100:] = low
    x[5, :8000] = low
    x[6] = np.nan
    x[7, 1::2] = np.nan
    x[8] = np.where(np.arange(9000) % 7 == 3, -0.0, 0.0)
    ids = np.tile([[0, 8999, 5000]], (9, 1))
    got = run(x, ids, top=32)
    check(x, got, ids, 32)
    assert bool(torch.isneginf(got[0][0]).all()) and float(got[1][0]) == 0
    assert got[2][0].tolist() == list(range(32)) == got[2][6].tolist() == got[2][8].tolist()


@pytest.mark.parametrize("order", ["up", "down", "blocks"])
@pytest.mark.parametrize("top", [1, 7, 32])
def test_sorted_rows(order, top):
    """The most likely tokens all in one place, in rising and falling order."""
    x = np.sort(logits(2, 70000, 5, True), -1)
    if order == "down":
        x = np.ascontiguousarray(x[:, ::-1])
    elif order == "blocks":
        x = np.ascontiguousarray(x.reshape(2, 70, 1000)[:, ::-1].reshape(2, 70000))
    check(x, run(x, [[1], [69999]], top=top), [[1], [69999]], top)


def test_large_and_close_logits():
    x = logits(4, 5000, 6, True)
    x[0] *= 1000
    x[1] += 1e4
    x[2] *= 1e-6
    x[3, 44] = 80.0                                         # one token nearly certain
    check(x, run(x, [[44]] * 4, top=8), [[44]] * 4, 8)
    x = np.zeros((1, 3), np.float32)
    x[0] = 3e38, -3e38, 1.0
    lp, h, ids, tl = run(x, [[0, 1, 2]], top=3)
    assert lp[0].tolist()[0] == 0.0 and lp[0].tolist()[1] == -np.inf and ids[0].tolist() == [0, 2, 1]


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -120, 0.1, 0.5])
@pytest.mark.parametrize("V", [4, 9000])
def test_logits_whose_difference_fp32_does_not_hold(scale, V):
    """3e38 and -3e38: 6e38 apart, which a scale below 1 may bring back."""
    x = np.full((4, V), -np.inf, np.float32)
    x[0, [0, 1, 2]] = 3e38, -3e38, 1.0
    x[1, [V - 1, 0, 1]] = 3e38, -3.4e38, 3e38
    x[2, :2] = -3.4e38
    x[3, [0, V - 1]] = -3.4e38, 3.4e38
    ids = np.tile([[0, 1, V - 1]], (4, 1))
    check(x, run(x, ids, top=3, scale=scale), ids, 3, scale)


def test_strides_shapes_and_what_was_not_asked_for():
    x = logits(7, 1003, 7, False)
    buf = torch.full((7, 2051), float("nan"), dtype=torch.float16, device="cuda")
    v = buf[:, 5:1008]
    v.copy_(torch.from_numpy(x))
    ids = np.arange(7) * 100
    got = tq.tq_logprobs(v, torch.from_numpy(ids.astype(np.int32)).cuda(), top=4, want_entropy=True)
    assert got[0].shape == (7,)
    check(x, got, ids, 4)
    same = torch.from_numpy(x).cuda()
    assert all(torch.equal(a, b) for a, b in zip(got, tq.tq_logprobs(same, torch.from_numpy(ids.astype(np.int32)).cuda(),
                                                                     top=4, want_entropy=True)))
    only = tq.tq_logprobs(same, top=4)
    assert only[0] is None and only[1] is None and torch.equal(only[2], got[2]) and torch.equal(only[3], got[3])
    only = tq.tq_logprobs(same, want_entropy=True)
    assert torch.equal(only[1], got[1]) and only[2] is None and only[3] is None
    assert torch.equal(tq.tq_logprobs(same[1::2], torch.from_numpy(ids[1::2].astype(np.int32)).cuda())[0], got[0][1::2])


def test_tokens_outside_the_vocabulary():
    x = logits(3, 500, 8, True)
    ids = np.array([[0, -1], [500, 499], [2 ** 31 - 1, -(2 ** 31)]])
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(x, run(x, ids, d_err=err), ids)
    assert int(err) == 4


def test_many_given_tokens():
    x = logits(2, 20000, 9, True)
    ids = np.random.default_rng(9).integers(0, 20000, (2, 1024))
    check(x, run(x, ids, top=3), ids, 3)


def test_rows_past_32_bits():
    """Rows whose first element lies beyond 2^32 bytes and 2^31 elements."""
    buf = torch.zeros(2 * (1 << 31) + 70000, dtype=torch.float16, device="cuda")
    v = buf.as_strided((2, 60000), ((1 << 32) + 8, 1))
    x = logits(2, 60000, 10, False)
    v.copy_(torch.from_numpy(x))
    ids = torch.tensor([5, 59999], dtype=torch.int32, device="cuda")
    check(x, tq.tq_logprobs(v, ids, top=6, want_entropy=True), [5, 59999], 6)


def test_the_same_bits_every_time_and_in_a_graph():
    x = torch.from_numpy(logits(3, 131072, 11, True)).cuda()
    ids = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    call = lambda **kw: tq.tq_logprobs(x, ids, top=20, want_entropy=True, **kw)
    want = call()
    need = tq.tq_logprobs_workspace_bytes(3, 131072, 1, 20)
    assert need > tq.WORKSPACE_COUNT_BYTES and tq.tq_logprobs_workspace_bytes(3, 4096, 1, 20) == 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:tq.WORKSPACE_COUNT_BYTES] = 0
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(call(workspace=ws), want))
        assert bool((ws[:tq.WORKSPACE_COUNT_BYTES] == 0).all())
    with pytest.raises(tq.TqError):
        call(workspace=ws[:need - 16].clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = call()
        big = torch.from_numpy(logits(300, 131072, 12, False)).cuda()
        held = []
        for i in range(3):
            x.copy_(torch.from_numpy(logits(3, 131072, 20 + i, True)))
            want = call()
            tq.tq_logprobs(big, top=5)                      # a larger buffer of the stream's
            held.append(torch.full((64 << 20,), 0x5A, dtype=torch.uint8, device="cuda"))
            g.replay()
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), i
            assert all(bool((t == 0x5A).all()) for t in held)
    torch.cuda.current_stream().wait_stream(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, call()))


def test_refusals():
    x = torch.zeros((2, 50), device="cuda")
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    for a, kw in (((x.double(),), {}), ((x.cpu(),), {}), ((x[0],), {}), ((x[:, ::2],), {}), ((x, ids.long()), {}),
                  ((x, ids[:1]), {}), ((x, ids[None]), {}), ((x, ids.cpu()), {}), ((x,), dict(d_err=ids)),
                  ((x,), dict(top=1 << 40))):
        with pytest.raises(ValueError):
            tq.tq_logprobs(*a, **kw)
    for kw, status in ((dict(top=33), 4), (dict(top=-1), 2), (dict(scale=0.0), 2), (dict(scale=-1.0), 2),
                       (dict(scale=float("inf")), 2), (dict(scale=float("nan")), 2)):
        with pytest.raises(tq.TqError) as e:
            tq.tq_logprobs(x, ids, **kw)
        assert e.value.status == status, kw
    for bad in (x[:, :5], x[:0], x[:, :0]):
        with pytest.raises(tq.TqError) as e:
            tq.tq_logprobs(bad, top=6)
        assert e.value.status == 2
    with pytest.raises(tq.TqError) as e:
        tq.tq_logprobs(x, torch.zeros((2, 1025), dtype=torch.int32, device="cuda"))
    assert e.value.status == 4
