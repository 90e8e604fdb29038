"""The parts that attention with sinks or over shared prefixes is cut into, from
the sizes of its workspace (CPU): a launch of all of them fits a grid, which holds
fewer than 2^32 threads, however many rows, heads and tokens there are."""

import ctypes
import itertools

import pytest

from paper_2609_09240_amd import tq

SOME = 1 << 20   # an address; nothing is read there
SIZES = list(itertools.product((1, 300, 65535), (1, 8, 32, 128), (10, 12, 20, 24, 26, 28, 30)))


def parts(rows, H, D, tokens, window=0, **scope):
    """Parts of a query (0: attended row by row as without a scope), one query a row and
    one query head a key/value head, over slots of up to `tokens` tokens."""
    c = tq.TqKvCache(1, H, D, 32, 1024, 1, tokens // 1024, 0, 1000, SOME, SOME, SOME, SOME)
    a = tq.TqKvAttn(rows, rows, 1, H, 0, window, 1.0, 0, SOME)
    s = tq.TqKvScope(**scope, cu_rows=SOME, prefix=SOME)
    n = tq.lib().tq_kv_attention_scope_workspace_bytes(ctypes.byref(c), ctypes.byref(a), ctypes.byref(s))
    return max(n - tq.WORKSPACE_COUNT_BYTES, 0) / (rows * H * (D + 4) * 4)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_sinks(D):
    most = 0
    for rows, H, log in SIZES:
        n = parts(rows, H, D, 1 << log, window=1 << log, sinks=4)
        assert n == int(n) and rows * H * n * 256 < 1 << 32, (rows, H, log, n)   # workgroups of 256 threads or 512
        most = max(most, n)
    assert most > 16   # some of them are in many


@pytest.mark.parametrize("D", [64, 128, 256])
def test_shared_prefixes(D):
    """A prefix of one record, which is one part: the others are the rows' own tokens."""
    together = 0
    for (rows, H, log), groups in itertools.product(SIZES, (1, 7)):
        if groups > rows or H == 128:
            continue
        n = parts(rows, H, D, 1 << log, n_groups=groups, max_prefix=32)
        if n == int(n) > 0:   # (attended together; a workspace of rows attended one by one has other sizes)
            tiles = (rows + 15) // 16 + groups - 1
            assert (rows * (n - 1) + tiles) * H * 256 < 1 << 32, (rows, H, log, groups, n)
            together += 1
    assert together > 20
