"""The binding of the paged cache's calls against a stand-in library and cache (CPU only)."""
import contextlib
import types

import pytest
import torch

from paper_2602_07160_gb300 import fem

S, H, PAGE, D = 2, 2, 16, 64


class Library:
    """Takes every call and does nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(fem, "load", lambda: lib)
    return lib


def stand_in(index=-1):
    """What the calls look at of a PagedCache; a host tensor's device index is -1."""
    return types.SimpleNamespace(index=index, device=torch.device("cpu"), H=H, d=D, page_size=PAGE, num_pages=4,
                                 row_dtype=torch.bfloat16, _ref=0)


def calls(cache, stream):
    """The three calls, each with tensors that pass the binding's other checks."""
    rows = torch.zeros((3, H, D), dtype=torch.bfloat16)
    table = torch.zeros((S, 1), dtype=torch.int32)
    lens, offsets = torch.zeros(S, dtype=torch.int32), torch.zeros(S + 1, dtype=torch.int32)
    return {"fem_cache_write": lambda: fem.fem_cache_write(cache, rows, rows, torch.zeros(3, dtype=torch.int64), stream=stream),
            "fem_cache_gather": lambda: fem.fem_cache_gather(cache, table, lens, offsets, 3, stream=stream),
            "fem_paged_read": lambda: fem.fem_paged_read(rows, cache, None, offsets, lens, table, max_q=1, stream=stream)}


@pytest.mark.parametrize("name", ["fem_cache_write", "fem_cache_gather", "fem_paged_read"])
def test_another_current_device_is_refused(library, monkeypatch, name):
    """The library launches on the current device: a cache of another one never reaches it."""
    stream = types.SimpleNamespace(cuda_stream=0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current"):
        calls(stand_in(), stream)[name]()
    assert library.calls == []


@pytest.mark.parametrize("name,outputs", [("fem_cache_gather", 2), ("fem_paged_read", 2)])
def test_outputs_are_memory_of_the_stream_that_writes_them(library, monkeypatch, name, outputs):
    """Memory of the current stream could still be in use there, or be given out again there, while the
    call's own stream writes it."""
    side, main = types.SimpleNamespace(cuda_stream=5), types.SimpleNamespace(cuda_stream=0)
    inside, made, recorded = [main], [], []

    @contextlib.contextmanager
    def use(stream):
        inside.append(stream)
        yield
        inside.pop()

    empty = torch.empty

    def allocate(*args, **kw):
        made.append(inside[-1])
        return empty(*args, **kw)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: inside[-1])
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append(s), raising=False)
    calls(stand_in(), side)[name]()
    assert library.calls == [name]
    assert made == [side] * outputs and recorded == [main] * outputs
