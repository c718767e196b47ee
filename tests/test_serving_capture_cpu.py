"""What a recorded graph reads stays alive as long as the graph does (no GPU needed: the recording itself is left out)."""
import contextlib
import gc
import weakref

import pytest
import torch

from paper_2510_21270_amd import binding as b


class _Stream:
    def wait_stream(self, other):
        pass


class _Graph:
    replays = 0

    def replay(self):
        self.replays += 1


@pytest.fixture
def recording(monkeypatch):
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "CUDAGraph", _Graph)
    monkeypatch.setattr(torch.cuda, "graph", lambda g: contextlib.nullcontext())


class _Cache:
    def __init__(self):
        self.K = torch.zeros(4)


def _step():
    s = b.DecodeStep.__new__(b.DecodeStep)
    s.cache, s.O = _Cache(), torch.zeros(1)
    return s


def _pipeline():
    return b.Pipeline(b.problem(batch=1, h_q=2, h_kv=1, n=256, d=128, block=128, segment=256, dtype="bf16", tau=0.9), device="cpu")


def _inputs(n):
    return [torch.zeros(8) for _ in range(n)]


@pytest.mark.parametrize("make,n", [(_pipeline, 6), (_step, 7)])
def test_a_recorded_graph_keeps_its_tensors(recording, monkeypatch, make, n):
    owner = make()
    monkeypatch.setattr(owner, "run", lambda *a: owner.O)
    args = _inputs(n)
    if make is _pipeline:
        args[4] = _Cache()
    refs = [weakref.ref(x) for x in args]
    owner.capture(*args)
    del args
    gc.collect()
    assert all(r() is not None for r in refs)
    owner.replay()
    assert owner.graph.replays == 1
    owner.capture(*_inputs(n))                             # the next recording lets them go
    gc.collect()
    assert all(r() is None for r in refs)


@pytest.mark.parametrize("make,n", [(_pipeline, 6), (_step, 7)])
@pytest.mark.parametrize("fails", ["before", "while"])
def test_a_recording_that_fails_leaves_the_former_one(recording, monkeypatch, make, n, fails):
    owner, first = make(), torch.zeros(1)
    monkeypatch.setattr(owner, "run", lambda *a: first)
    args = _inputs(n)
    refs = [weakref.ref(x) for x in args]
    owner.capture(*args)
    graph = owner.graph
    del args
    calls = []

    def run(*a):
        calls.append(1)
        if len(calls) == (1 if fails == "before" else 2):
            raise b.PbsError("refused")
        return torch.zeros(1)

    monkeypatch.setattr(owner, "run", run)
    with pytest.raises(b.PbsError, match="refused"):
        owner.capture(*_inputs(n))
    gc.collect()
    assert owner.graph is graph and all(r() is not None for r in refs)
    assert owner.replay() is (first if make is _pipeline else owner.O) and graph.replays == 1
