"""Eviction's host side without a GPU."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2609_32046_gb300 import binding
from test_budget_host import Spy, cache, receiver


def test_memory_comes_from_the_streams_own(monkeypatch):
    """What a call on a stream allocates is that stream's: another stream's next allocation would get the memory while
    the call still uses it."""
    names = {"pool": SimpleNamespace(cuda_stream=64), "default": SimpleNamespace(cuda_stream=0)}
    monkeypatch.setattr(torch.cuda, "Stream", SimpleNamespace)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: ("on", s))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: ("external", handle, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: names["default"])
    x = SimpleNamespace(device=torch.device("cuda", 3), is_cuda=True)
    for current in (0, 32, 64):
        monkeypatch.setattr(binding, "_raw_stream", lambda index, current=current: current)
        for stream, handle, want in ((names["pool"], 64, names["pool"]), (64, 64, ("external", 64, x.device)), (0, 0, names["default"])):
            got = binding._memory_for(stream, x)
            if handle == current:
                assert isinstance(got, contextlib.nullcontext)
            else:
                assert got == ("on", want)
        assert isinstance(binding._memory_for(None, x), contextlib.nullcontext)
        assert isinstance(binding._memory_for(64, torch.zeros(1)), contextlib.nullcontext)


@pytest.mark.parametrize("stream", [None, 64])
def test_evict_allocates_there(monkeypatch, stream):
    inside, made, empty = [], [], torch.empty

    @contextlib.contextmanager
    def memory_for(s, tensor):
        inside.append(s)
        yield
        inside.append("left")

    def allocate(*args, **kw):
        made.append(list(inside))
        return empty(*args, **kw)

    monkeypatch.setattr(binding, "_memory_for", memory_for)
    monkeypatch.setattr(binding, "_stream_on", lambda s, x: s or 0)
    monkeypatch.setattr(torch, "empty", allocate)
    caches, w = [cache(40), cache(30)], [torch.zeros(3, 2, 40)] * 2
    rx = receiver(Spy())
    idx = rx.evict(caches, w, 9, stream=stream)
    assert [tuple(x.shape) for x in idx] == [(3, 2, 9)] * 2 and made == [[stream]] * 2
    rx.evict(caches, w, 9, idx=idx, stream=stream)
    assert len(made) == 2
