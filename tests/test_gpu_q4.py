"""Products with 4-bit weights against the fp64 oracle (GPU).

Quantising and unpacking are unique results and compared bit for bit.  The
product's terms are exact and only its fp32 sums round: with u = 2^-24 the
error of n additions in any order is at most n u sum|terms|; a fused multiply
adds one rounding more, and the matrix cores are allowed twice the rounding of
an addition, so 2 (K + 64) u of the terms bounds it.  Cases whose sums are
exact (small whole numbers) must be equal, which no misplaced element
survives.
"""

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2609_09240_amd import tq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _upload(codes, s, m, group):
    n, k = codes.shape
    cb, pb = q4.pack_matrix(codes, s, m, group)
    return tq.Q4Linear(n, k, group, torch.from_numpy(cb).cuda(), torch.from_numpy(pb).cuda())


def _random(n, k, group, seed):
    r = np.random.default_rng(seed)
    ng = -(-k // group)
    s = r.uniform(0.002, 0.02, (n, ng)).astype(np.float16)
    return (r.integers(0, 16, (n, k)).astype(np.uint8), s,
            (-7.5 * s.astype(np.float64) + r.standard_normal((n, ng)) * 0.002).astype(np.float16))


@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (16, 128, 128), (17, 129, 32), (5, 300, 64), (40, 1000, 128),
                                       (33, 4096, 64), (130, 31, 128)])
def test_quantize_and_unpack_are_the_oracles(n, k, group):
    r = np.random.default_rng(n * 7 + k)
    w = r.standard_normal((n, k)).astype(np.float16)
    w[0, :min(k, 3)] = 0.0
    if k > 40:
        w[-1, 32:40] = 60000.0
        w[-1, 1] = -60000.0
    codes, s, m = q4.quantise(w, group)
    mat = tq.tq_q4_quantize(torch.from_numpy(w).cuda(), group)
    cb, pb = q4.pack_matrix(codes, s, m, group)
    np.testing.assert_array_equal(mat.codes.cpu().numpy(), cb)
    np.testing.assert_array_equal(mat.params.cpu().numpy().view(np.uint16) & 0x7FFF, pb.view(np.uint16) & 0x7FFF)
    at = np.arange(k) // group
    want = (codes.astype(np.float32) * s.astype(np.float32)[:, at] + m.astype(np.float32)[:, at]).astype(np.float16)
    np.testing.assert_array_equal(tq.tq_q4_unpack_fp16(mat).cpu().numpy(), want)


def test_quantize_groups_that_are_not_finite():
    w = np.ones((3, 200), np.float16)
    w[:, ::2] = 2.0
    w[0, 5], w[1, 100], w[2, 199] = np.inf, np.nan, -np.inf
    codes, s, m = q4.quantise(w, 64)
    got = tq.tq_q4_unpack_fp16(tq.tq_q4_quantize(torch.from_numpy(w).cuda(), 64)).cpu().numpy()
    at = np.arange(200) // 64
    np.testing.assert_array_equal(np.isnan(got), np.isnan(s)[:, at])
    np.testing.assert_array_equal(got[~np.isnan(got)], w[~np.isnan(got)])


def test_quantize_reads_strided_rows():
    w = torch.randn((20, 512), dtype=torch.float16, device="cuda")
    a = tq.tq_q4_quantize(w[:, 3:260], 32)
    b = tq.tq_q4_quantize(w[:, 3:260].contiguous(), 32)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.params, b.params)


@pytest.mark.parametrize("B", [1, 2, 5, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (15, 100, 64), (16, 128, 128), (100, 1152, 32), (257, 1000, 64),
                                       (48, 2177, 128)])
def test_exact_sums_are_equal(n, k, group, B):
    """Whole inputs and offsets, scales that are powers of two: every partial
    sum is a whole multiple of 1/4 below 2^22, exact in fp32 in any order."""
    r = np.random.default_rng(B * 1000 + n)
    ng = -(-k // group)
    codes = r.integers(0, 16, (n, k)).astype(np.uint8)
    s = r.choice([0.25, 0.5, 1.0, -0.5], (n, ng)).astype(np.float16)
    m = r.integers(-8, 9, (n, ng)).astype(np.float16)
    x = r.integers(-3, 4, (B, k)).astype(np.float16)
    y = tq.tq_q4_gemm(_upload(codes, s, m, group), torch.from_numpy(x).cuda(), out_f32=True)
    np.testing.assert_array_equal(y.cpu().numpy().astype(np.float64), q4.gemm(codes, s, m, group, x))


@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("n,k,B,group", [(1024, 4096, 1, 128), (300, 5000, 5, 32), (4096, 1024, 16, 64),
                                         (70, 12288, 24, 128), (33000, 256, 3, 64), (511, 3001, 64, 32),
                                         (33000, 130, 40, 128), (1, 16384, 1, 128)])
def test_products_within_the_bound(n, k, B, group, out_f32):
    codes, s, m = _random(n, k, group, n + k)
    x = np.random.default_rng(B).standard_normal((B, k)).astype(np.float16)
    mat, xd = _upload(codes, s, m, group), torch.from_numpy(x).cuda()
    got = tq.tq_q4_gemm(mat, xd, out_f32=out_f32)
    assert torch.equal(got, tq.tq_q4_gemm(mat, xd, out_f32=out_f32))
    want = q4.gemm(codes, s, m, group, x)
    bound = 2 * (k + 64) * U * q4.gemm_scale(codes, s, m, group, x)
    if not out_f32:
        bound = bound * (1 + 2.0 ** -11) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
    err = np.abs(got.cpu().numpy().astype(np.float64) - want)
    assert (err <= bound).all(), float((err / bound).max())
    if out_f32:
        # rounding errors of both signs: far below the worst case
        assert np.linalg.norm(err) <= 64 * U * np.linalg.norm(q4.gemm_scale(codes, s, m, group, x))


def test_rows_do_not_depend_on_each_other():
    codes, s, m = _random(200, 700, 64, 3)
    mat = _upload(codes, s, m, 64)
    x = torch.randn((16, 700), dtype=torch.float16, device="cuda")
    y = tq.tq_q4_gemm(mat, x, out_f32=True)
    x2 = x.clone()
    x2[1:] = float("nan")
    assert torch.equal(tq.tq_q4_gemm(mat, x2, out_f32=True)[0], y[0])
    assert torch.equal(tq.tq_q4_gemm(mat, x[3], out_f32=True), y[3])


@pytest.mark.parametrize("offset", [1, 3, 8])
def test_inputs_anywhere_and_with_strides(offset):
    codes, s, m = _random(90, 777, 32, 5)
    mat = _upload(codes, s, m, 32)
    buf = torch.full((6, 900), float("nan"), dtype=torch.float16, device="cuda")
    x = buf[:, offset:offset + 777]
    x.copy_(torch.randn((6, 777), device="cuda"))
    assert torch.equal(tq.tq_q4_gemm(mat, x, out_f32=True), tq.tq_q4_gemm(mat, x.contiguous(), out_f32=True))


def test_outputs_that_are_not_finite():
    """An infinite input gives an infinity under every weight that is not 0,
    NaN under a weight of 0; NaN inputs and parameters give NaN."""
    codes, s, m = _random(40, 300, 64, 9)
    codes[3, 7], m[3, 0] = 0, 0.0                       # a weight of 0
    s[5, 4] = np.nan
    x = np.random.default_rng(4).standard_normal((3, 300)).astype(np.float16)
    x[1, 7] = np.inf
    x[2, 290] = np.nan
    got = tq.tq_q4_gemm(_upload(codes, s, m, 64), torch.from_numpy(x).cuda(), out_f32=True).cpu().numpy()
    with np.errstate(invalid="ignore"):
        w = q4.values(codes, s, m, 64)
        want = x.astype(np.float64) @ w.T
    assert np.isnan(want[1, 3]) and np.isinf(want[1]).sum() == 38
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    np.testing.assert_array_equal(got[inf], want[inf])


@pytest.mark.parametrize("n,k,B,group", [(100, 4096, 17, 64), (1000, 5000, 40, 32), (4096, 2048, 64, 128),
                                         (33000, 1024, 64, 64), (16, 16384, 32, 128)])
def test_split_along_k(n, k, B, group):
    """Parts of K joined in one launch: exact sums are equal with and without
    a workspace, and a workspace serves call after call and other shapes."""
    r = np.random.default_rng(n)
    ng = -(-k // group)
    codes = r.integers(0, 16, (n, k)).astype(np.uint8)
    s = r.choice([0.25, 0.5, -0.5], (n, ng)).astype(np.float16)
    m = r.integers(-8, 9, (n, ng)).astype(np.float16)
    x = r.integers(-1, 2, (B, k)).astype(np.float16)
    mat, xd = _upload(codes, s, m, group), torch.from_numpy(x).cuda()
    want = q4.gemm(codes, s, m, group, x)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    for b in (B, 17, B):
        for kw in (dict(workspace=ws), dict()):
            y = tq.tq_q4_gemm(mat, xd[:b], out_f32=True, **kw)
            np.testing.assert_array_equal(y.cpu().numpy().astype(np.float64), want[:b])
    y = torch.empty((B, n), dtype=torch.float32, device="cuda")
    tq._check(tq.lib().tq_q4_gemm(mat._ref, xd.data_ptr(), k, B, y.data_ptr(), 1, None, 0, tq._stream(None)), "gemm")
    np.testing.assert_array_equal(y.cpu().numpy().astype(np.float64), want)


def test_split_along_k_from_a_graph():
    codes, s, m = _random(300, 4096, 64, 2)
    mat = _upload(codes, s, m, 64)
    x = torch.randn((40, 4096), dtype=torch.float16, device="cuda")
    y = torch.empty((40, 300), dtype=torch.float16, device="cuda")
    tq.tq_q4_gemm(mat, x, Y=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tq.tq_q4_gemm(mat, x, Y=y)
    for i in range(4):
        x.copy_(torch.randn((40, 4096), device="cuda"))
        want = tq.tq_q4_gemm(mat, x)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


def test_on_another_stream():
    codes, s, m = _random(64, 512, 128, 1)
    mat = _upload(codes, s, m, 128)
    x = torch.randn((4, 512), dtype=torch.float16, device="cuda")
    y = tq.tq_q4_gemm(mat, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z = tq.tq_q4_gemm(mat, x, stream=side)
    q = tq.tq_q4_quantize(tq.tq_q4_unpack_fp16(mat, stream=side), 128, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, z)
    r = tq.tq_q4_quantize(tq.tq_q4_unpack_fp16(mat), 128)
    assert torch.equal(q.codes, r.codes) and torch.equal(q.params, r.params)


def test_replayed_from_a_graph():
    codes, s, m = _random(500, 1024, 64, 2)
    mat = _upload(codes, s, m, 64)
    x = torch.randn((2, 1024), dtype=torch.float16, device="cuda")
    y = torch.empty((2, 500), dtype=torch.float16, device="cuda")
    tq.tq_q4_gemm(mat, x, Y=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tq.tq_q4_gemm(mat, x, Y=y)
    for i in range(4):
        x.copy_(torch.randn((2, 1024), device="cuda"))
        want = tq.tq_q4_gemm(mat, x)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


def test_refusals():
    mat = _upload(*_random(32, 256, 64, 1), 64)
    x = torch.zeros((65, 256), dtype=torch.float16, device="cuda")
    with pytest.raises(tq.TqError) as e:
        tq.tq_q4_gemm(mat, x)
    assert e.value.status == 2
    assert tq.tq_q4_workspace_bytes(mat, 16) == 0 and tq.tq_q4_workspace_bytes(mat, 65) == 0
    deep = tq.Q4Linear.empty(32, 4096, 64)
    wide = torch.zeros((64, 4096), dtype=torch.float16, device="cuda")
    for ws in (torch.zeros(tq.tq_q4_workspace_bytes(deep, 64) - 16, dtype=torch.uint8, device="cuda"),):
        with pytest.raises(tq.TqError) as e:
            tq.tq_q4_gemm(deep, wide, workspace=ws)
        assert e.value.status == 2
    for bad in (x[:2].float(), x[:2, :100], x[:2].t(), x[:2].cpu()):
        with pytest.raises(ValueError):
            tq.tq_q4_gemm(mat, bad)
    with pytest.raises(ValueError):
        tq.tq_q4_gemm(mat, x[:2], Y=torch.empty((2, 31), dtype=torch.float16, device="cuda"))
    with pytest.raises(tq.TqError):
        tq.Q4Linear.empty(4, 4, group=16)
    with pytest.raises(ValueError):
        tq.Q4Linear(32, 257, 64, mat.codes, mat.params)
