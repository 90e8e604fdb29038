"""The binding's choice of a workspace, with the stream and its capture state
replaced: a captured call never gets, and never leaves behind, a buffer that
an eager call uses, since a graph outlives the handle's hold on it."""

import os
import re

import pytest
import torch

from paper_2609_09240_amd import tq


class Streams:
    """What the binding asks torch for."""

    def __init__(self, monkeypatch):
        self.current, self.capturing = 1, False
        monkeypatch.setattr(tq, "_stream", lambda stream: self.current)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)


@pytest.fixture
def streams(monkeypatch):
    return Streams(monkeypatch)


def test_eager_calls_share_one_buffer_a_stream(streams):
    ws = tq._Workspaces("cpu")
    a = ws.get(40000, None)
    assert a.numel() >= 40000 and ws.get(100, None) is a
    streams.current = 2
    b = ws.get(100, None)
    assert b is not a and ws.get(50, None) is b
    streams.current = 1
    c = ws.get(50000, None)
    assert c is not a and ws.get(40000, None) is c


@pytest.mark.parametrize("need", [100, 40000, 60000])
def test_a_captured_call_has_a_buffer_of_its_own(streams, need):
    """Warmed up and captured on the same stream, with a buffer there that
    is large enough and one that is not."""
    ws = tq._Workspaces("cpu")
    warm = ws.get(40000, None)
    kept = dict(ws.by_stream)
    streams.capturing = True
    got = [ws.get(need, None) for _ in range(3)]
    assert len({t.data_ptr() for t in got + [warm]}) == 4
    assert all(t.numel() >= need for t in got)
    streams.capturing = False
    # The handle holds what it held, and no eager call meets a graph's buffer.
    assert ws.by_stream == kept and ws.get(40000, None) is warm
    assert ws.get(80000, None).data_ptr() not in {t.data_ptr() for t in got}


def test_a_capture_on_a_stream_that_was_never_used(streams):
    ws = tq._Workspaces("cpu")
    streams.capturing = True
    a, b = ws.get(64, None), ws.get(64, None)
    assert a is not b and not ws.by_stream


@pytest.mark.parametrize("need", [100, 16384, 50000])
def test_counts_are_zeros(streams, monkeypatch, need):
    """Whatever the memory held before, the counts at its front are zeros."""
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).fill_(0xA5))
    for streams.capturing in (False, True):
        t = tq._Workspaces("cpu").get(need, None)
        assert bool((t[:tq.WORKSPACE_COUNT_BYTES] == 0).all())


def test_the_header_says_the_same():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tq.h")
    with open(path) as f:
        n = re.search(r"#define TQ_WORKSPACE_COUNT_BYTES (\d+)", f.read())
    assert int(n.group(1)) == tq.WORKSPACE_COUNT_BYTES
