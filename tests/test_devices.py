"""Calls of the operators around a decode step with one tensor of another device
than the current one (CPU: tensors that say where they are, and a library that
notes its calls): each of them is refused before the library is called."""

import pytest
import torch

from paper_2609_09240_amd import tq

HERE, ELSEWHERE = 0, 1


class Placed(torch.Tensor):
    """A tensor on the GPU, as far as the binding can see."""
    is_cuda = property(lambda t: True)

    def get_device(self):
        return getattr(self, "at", HERE)


def placed(t, at=HERE):
    t = t.as_subclass(Placed)
    t.at = at
    return t


class Calls:
    """The library: sizes as they are, calls noted only."""

    def __init__(self, real):
        self.real, self.made = real, []

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 1 << 20
        if name.endswith("page_bytes"):
            return getattr(self.real, name)
        return lambda *a: self.made.append(name) or 0


@pytest.fixture
def calls(monkeypatch):
    c = Calls(tq.lib())
    monkeypatch.setattr(tq, "lib", lambda: c)
    monkeypatch.setattr(tq, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: HERE)
    return c


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def f16(*shape):
    return torch.zeros(shape, dtype=torch.float16)


WS = torch.zeros(1 << 20, dtype=torch.uint8)

ROPE = dict(q=f16(3, 4, 64), k=f16(3, 2, 64), positions=torch.zeros((2, 3), dtype=torch.int32), freq=torch.ones(32),
            axis=torch.zeros(32, dtype=torch.uint8), q_out=f16(3, 4, 64), k_out=f16(3, 2, 64))
LOGPROBS = dict(logits=torch.zeros(3, 50), ids=i32(1, 2, 3), d_err=i32(0), workspace=WS)
ATTENTION = dict(q=f16(3, 4, 64), seqs=i32(0, 1, 2), cu_q=i32(0, 1, 2, 3), o=f16(3, 4, 64), lse=torch.zeros(3, 4),
                 workspace=WS, prefix=i32(32, 32, 32), groups=i32(0, 3))
SINKS = {k: v for k, v in ATTENTION.items() if k not in ("prefix", "groups")}
PREFIX = dict(seqs=i32(0, 1, 2), groups=i32(0, 3), prefix=i32(0, 0, 0))
BUFFERS = ("data", "pages", "lens", "refs")


def cache(at):
    b = dict(data=torch.zeros((1, 4, 2 * 32 * (64 + 8)), dtype=torch.uint8), pages=torch.zeros((3, 2), dtype=torch.int32),
             lens=torch.zeros(3, dtype=torch.int32), refs=torch.zeros(4, dtype=torch.int32))
    return tq.KVCache(*[placed(b[n], ELSEWHERE if n == at else HERE) for n in BUFFERS], 2, 64, 32, 64)


def run(name, tensors, at=None):
    """A call with all its tensors here, but for `at`."""
    t = {n: placed(x.clone(), ELSEWHERE if n == at else HERE) for n, x in tensors.items()}
    if name == "rope":
        return tq.tq_rope(**t)
    if name == "logprobs":
        return tq.tq_logprobs(**t, top=2, want_entropy=True)
    c = cache(at)
    if name == "shared_prefix":
        return tq.tq_kv_shared_prefix(c, **t)
    return tq.tq_kv_attention(c, 0, **t, max_q=1, **(dict(window=5, sinks=2) if name == "sinks" else {}))


FORMS = [("rope", ROPE, ()), ("logprobs", LOGPROBS, ()), ("prefix", ATTENTION, BUFFERS), ("sinks", SINKS, BUFFERS),
         ("shared_prefix", PREFIX, BUFFERS)]


@pytest.mark.parametrize("name,tensors", [f[:2] for f in FORMS])
def test_all_of_them_here(calls, name, tensors):
    run(name, tensors)
    assert len(calls.made) == 1


@pytest.mark.parametrize("name,tensors,at", [(n, t, at) for n, t, more in FORMS for at in (*t, *more)],
                         ids=lambda x: x if isinstance(x, str) else "")
def test_one_of_them_elsewhere(calls, name, tensors, at):
    with pytest.raises(ValueError, match="current device"):
        run(name, tensors, at)
    assert calls.made == []
