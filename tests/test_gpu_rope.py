"""Rotary positions against the fp64 oracle (GPU).

Tolerance.  An angle in turns is rounded to fp32 (2^-25 of at most half a turn:
2^-23.3 radians), sine and cosine to about 2^-23 each with their scale; two
products, a sum: together at most 2^-20 of scale (|x1| + |x2|).  Then one rounding
to fp16: 2^-11 of the value, 2^-25 below its normal numbers.
"""

import numpy as np
import pytest
import torch

from oracle import decode
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu


def _x(shape, seed):
    return np.random.default_rng(seed).standard_normal(shape).astype(np.float16)


def _freq(n):
    return (10000.0 ** (-np.arange(n) / n)).astype(np.float32)


def check(got, x, pos, freq, axis=None, adjacent=False, inverse=False, scale=1.0):
    want = decode.rope(x, pos, freq, axis, adjacent, inverse, scale)
    n = len(freq)
    size = np.zeros(x.shape)
    a = np.arange(n)
    i, j = (2 * a, 2 * a + 1) if adjacent else (a, a + n)
    s = np.abs(x[..., i].astype(np.float64)) + np.abs(x[..., j].astype(np.float64))
    size[..., i] = size[..., j] = abs(scale) * s
    err = np.abs(got.cpu().numpy().astype(np.float64) - want)
    assert (err <= 2.0 ** -20 * size + 2.0 ** -11 * np.abs(want) * (size > 0) + 2.0 ** -25 * (size > 0)).all(), err.max()


def up(x, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


@pytest.mark.parametrize("D,rot", [(128, 128), (64, 64), (256, 256), (128, 32), (96, 24), (80, 80), (36, 12), (2, 2),
                                   (6, 2), (1024, 1022), (1023, 510), (130, 128)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("T,hq,hkv", [(1, 4, 2), (37, 5, 1), (300, 1, 0)])
def test_shapes(D, rot, adjacent, T, hq, hkv):
    q, k = _x((T, hq, D), D), _x((T, hkv, D), rot)
    f = _freq(rot // 2)
    pos = np.random.default_rng(T).integers(0, 5000, T).astype(np.int32)
    a, b = tq.tq_rope(up(q), up(k) if hkv else None, up(pos), up(f), adjacent=adjacent), None
    if hkv:
        a, b = a
        check(b, k, pos, f, adjacent=adjacent)
    check(a, q, pos, f, adjacent=adjacent)


@pytest.mark.parametrize("T,hq,hkv,D,rot", [(27000, 30, 9, 16, 16), (65537, 30, 9, 16, 16), (20011, 17, 6, 6, 2),
                                            (700, 5, 2, 1023, 510)])
def test_many_tokens(T, hq, hkv, D, rot):
    """Enough of them that one workgroup takes more heads than it loads at once."""
    q, k = _x((T, hq, D), D), _x((T, hkv, D), rot)
    f = _freq(rot // 2)
    pos = np.random.default_rng(T).integers(0, 100000, T).astype(np.int32)
    a, b = tq.tq_rope(up(q), up(k), up(pos), up(f))
    check(a, q, pos, f)
    check(b, k, pos, f)
    c = up(k)
    tq.tq_rope(c, None, up(pos), up(f), q_out=c)
    assert torch.equal(c, b)


@pytest.mark.parametrize("axes", [2, 3, 8])
@pytest.mark.parametrize("inverse", [False, True])
def test_axes(axes, inverse):
    q, k = _x((50, 14, 64), 1), _x((50, 2, 64), 2)
    r = np.random.default_rng(axes)
    pos = r.integers(-100, 100000, (axes, 50)).astype(np.int32)
    f = _freq(32)
    for axis in (np.arange(32) % axes, np.sort(r.integers(0, axes, 32)), np.full(32, axes - 1), r.integers(0, 256, 32)):
        axis = axis.astype(np.uint8)
        a, b = tq.tq_rope(up(q), up(k), up(pos), up(f), axis=up(axis), inverse=inverse, scale=0.75)
        check(a, q, pos, f, axis, inverse=inverse, scale=0.75)
        check(b, k, pos, f, axis, inverse=inverse, scale=0.75)


def test_far_positions_and_steep_frequencies():
    q = _x((7, 3, 64), 3)
    pos = np.array([0, 1, 10 ** 6, 2 ** 24 + 1, 2 ** 31 - 1, -(2 ** 31), -5], np.int32)
    f = np.concatenate([_freq(28), [0.0, 1.0, 0.1, -0.7]]).astype(np.float32)
    # 2^31 turns of a radian, rounded at 2^-53 of their number: 2^-22 turns more
    got = tq.tq_rope(up(q), None, up(pos), up(f))
    want = decode.rope(q, pos, f)
    s = np.abs(q[..., :32].astype(np.float64)) + np.abs(q[..., 32:].astype(np.float64))
    bound = 2.0 ** -19 * np.concatenate([s, s], -1) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
    assert (np.abs(got.cpu().numpy().astype(np.float64) - want) <= bound).all()


@pytest.mark.parametrize("rot", [128, 48, 20])
@pytest.mark.parametrize("adjacent", [False, True])
def test_strides_in_place_and_what_is_left_alone(rot, adjacent):
    """q and k inside the output of one projection, at odd addresses, turned in
    place; everything else there stays as it was."""
    T, hq, hkv, D = 29, 6, 2, 128
    buf = torch.from_numpy(_x((T, 10 * D + 7), 4)).cuda()
    f, pos = _freq(rot // 2), np.arange(1000, 1000 + T, dtype=np.int32)
    before = buf.clone()
    q = buf[:, 3:3 + hq * D].unflatten(1, (hq, D))
    k = buf[:, 3 + hq * D:3 + (hq + hkv) * D].unflatten(1, (hkv, D))
    xq, xk = q.cpu().numpy().copy(), k.cpu().numpy().copy()
    new = tq.tq_rope(q, k, up(pos), up(f), adjacent=adjacent)
    assert torch.equal(buf, before)
    got = tq.tq_rope(q, k, up(pos), up(f), adjacent=adjacent, q_out=q, k_out=k)
    assert got[0] is q and torch.equal(q, new[0]) and torch.equal(k, new[1])
    check(q, xq, pos, f, adjacent=adjacent)
    check(k, xk, pos, f, adjacent=adjacent)
    assert torch.equal(q[..., rot:], before[:, 3:3 + hq * D].unflatten(1, (hq, D))[..., rot:])
    same = torch.ones_like(buf, dtype=torch.bool)
    same[:, 3:3 + (hq + hkv) * D] = False
    assert torch.equal(buf[same], before[same])
    # one in place, the other not; outputs with strides
    wide = torch.full((T, hkv, 2 * D), 9.0, dtype=torch.float16, device="cuda")
    src = before[:, 3:3 + hq * D].unflatten(1, (hq, D))
    kin = before[:, 3 + hq * D:3 + (hq + hkv) * D].unflatten(1, (hkv, D))
    tq.tq_rope(src, kin, up(pos), up(f), adjacent=adjacent, q_out=src, k_out=wide[..., 5:5 + D])
    assert torch.equal(src, new[0]) and torch.equal(wide[..., 5:5 + D], new[1])
    assert bool((wide[..., :5] == 9).all()) and bool((wide[..., 5 + D:] == 9).all())


def test_inverse_is_the_gradient():
    """<g, R x> = <R' g, x> against the oracle, and a difference of the loss."""
    x, g = _x((9, 4, 64), 5), _x((9, 4, 64), 6)
    pos, f = np.arange(9, dtype=np.int32) * 77, _freq(24)
    dx = tq.tq_rope(up(g), None, up(pos), up(f), inverse=True, scale=1.5)
    check(dx, g, pos, f, inverse=True, scale=1.5)
    loss = lambda v: float((decode.rope(v, pos, f, scale=1.5) * g.astype(np.float64)).sum())
    e = np.zeros(x.shape)
    d = dx.cpu().numpy().astype(np.float64)
    for at in ((0, 0, 0), (3, 1, 23), (8, 3, 47), (5, 2, 60), (4, 0, 30)):
        e[at] = 1e-3
        # the map is linear: the difference is exact but for fp64 (1e-9) and dx's rounding to fp16
        slope = (loss(x + e) - loss(x - e)) / 2e-3
        size = 1.5 * np.abs(g[at[:2]].astype(np.float64)).max() * 2
        want = g[at].astype(np.float64) if at[2] >= 48 else slope
        assert abs(d[at] - want) <= 2.0 ** -11 * abs(want) + 2.0 ** -19 * size + 1e-8, at
        e[at] = 0


def test_special_values_stay_with_their_pair():
    x = _x((3, 2, 64), 7)
    x[1, 0, 5] = np.inf
    x[2, 1, 40] = np.nan
    got = tq.tq_rope(up(x), None, up(np.array([3, 4, 5], np.int32)), up(_freq(32))).cpu().numpy()
    bad = ~np.isfinite(got)
    want = np.zeros_like(bad)
    want[1, 0, [5, 37]] = want[2, 1, [8, 40]] = True
    assert (bad == want).all()


def test_streams_and_graphs():
    q, k = (torch.from_numpy(_x((100, h, 128), h)).cuda() for h in (8, 2))
    pos, f = torch.arange(100, dtype=torch.int32, device="cuda"), up(_freq(64))
    want = tq.tq_rope(q, k, pos, f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tq.tq_rope(q, k, pos, f, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    outs = [torch.empty_like(t) for t in (q, k)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tq.tq_rope(q, k, pos, f, q_out=outs[0], k_out=outs[1])
    for i in range(3):
        pos += 1000 * i
        q.copy_(torch.randn_like(q))
        want = tq.tq_rope(q, k, pos, f)
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i


def test_refusals():
    q, k = torch.zeros((4, 2, 64), dtype=torch.float16, device="cuda"), torch.zeros((4, 1, 64), dtype=torch.float16, device="cuda")
    pos, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    tq.tq_rope(q, k, pos, f)
    wide = torch.zeros((4, 2, 128), dtype=torch.float16, device="cuda")
    for a in ((q.float(), k, pos, f), (q.cpu(), k, pos, f), (wide[..., ::2], k, pos, f), (q, k[:3], pos, f),
              (q, wide[:, :1], pos, f), (q, k, pos[:3], f), (q, k, pos.long(), f), (q, k, pos, f.double()),
              (q, k, pos.expand(2, 4), f), (q[0], k, pos, f), (q, k, pos.cpu(), f)):
        with pytest.raises(ValueError):
            tq.tq_rope(*a)
    for kw in (dict(axis=torch.zeros(31, dtype=torch.uint8, device="cuda")), dict(axis=torch.zeros(32, device="cuda")),
               dict(q_out=q[:3]), dict(k_out=q), dict(q_out=q.float())):
        with pytest.raises(ValueError):
            tq.tq_rope(q, k, pos, f, **kw)
    for a, kw, status in (((q, k, pos, torch.ones(33, device="cuda")), {}, 2), ((q, k, pos, f), dict(scale=float("nan")), 2),
                          ((q, k, pos, torch.ones(0, device="cuda")), {}, 2),
                          ((q[:0], k[:0], pos[:0], f), {}, 2),
                          ((q, k, pos.expand(9, 4).contiguous(), f),
                           dict(axis=torch.zeros(32, dtype=torch.uint8, device="cuda")), 4)):
        with pytest.raises(tq.TqError) as e:
            tq.tq_rope(*a, **kw)
        assert e.value.status == status
    view = wide.flatten()[:4 * 2 * 64].view(4, 2, 64)
    other = wide.as_strided((4, 2, 64), (256, 128, 1))
    with pytest.raises(tq.TqError):                     # starts where the input does, with other strides
        tq.tq_rope(view, None, pos, f, q_out=other)
    with pytest.raises(tq.TqError):                     # a row that all tokens are written to
        tq.tq_rope(q, None, pos, f, q_out=torch.empty_like(q[:1]).expand(4, 2, 64))
