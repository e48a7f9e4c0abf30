"""On which GPU the 8-bit cache's binding calls the library: a stand-in library records the current
device, stand-in tensors and streams live on the second of two GPUs that are not there."""

import contextlib

import pytest
import torch

from paper_2607_01308_amd import _cabi as C
from paper_2607_01308_amd import qcache

HERE, THERE = torch.device("cuda", 0), torch.device("cuda", 1)


class Tensor(torch.Tensor):
    """A CPU tensor that says that it lives on another device."""
    device = property(lambda self: THERE)
    is_cuda = property(lambda self: True)

    def record_stream(self, s):
        assert s.device == THERE


def on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(Tensor)


class Stream:
    def __init__(self, device, handle):
        self.device, self.cuda_stream = device, handle


@pytest.fixture
def calls(monkeypatch):
    """(entry point, device current at the call, stream) of the calls that reach the library."""
    current, log = [0], []

    @contextlib.contextmanager
    def device(dev):
        current.append(torch.device(dev).index)
        yield
        current.pop()

    @contextlib.contextmanager
    def stream(s):
        with device(s.device):
            yield

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name != "cm_qcache_attention_size":
                    log.append((name, current[-1], args[-1]))
                return C.CM_OK
            return call

    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k).as_subclass(Tensor))
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[-1])
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda d=None: Stream(torch.device("cuda", current[-1] if d is None else d), 0))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(C, "lib", Library)
    return log


def three_calls(stream=None):
    cache = qcache.QCache(on_gpu(1, 2, 4, 2, 16, 64, dtype=torch.uint8), on_gpu(1, 2, 4, 2))
    table, one = on_gpu(1, 4, dtype=torch.int32), on_gpu(1, dtype=torch.int32)
    step = qcache.qcache_tables(4, 16, one, one, on_gpu(4, dtype=torch.int32), table, 1, stream=stream)
    qcache.qcache_write(cache, 0, on_gpu(1, 2, 64), on_gpu(1, 2, 64), step.slots, stream=stream)
    qcache.qcache_attention(cache, 0, on_gpu(1, 4, 64), table, step.lens, stream=stream)


NAMES = ["cm_qcache_tables", "cm_qcache_write", "cm_qcache_attention"]


def test_calls_are_made_on_the_caches_gpu(calls):
    three_calls()
    assert calls == [(name, 1, 0) for name in NAMES]
    assert torch.cuda.current_device() == 0
    calls.clear()
    three_calls(Stream(THERE, 77))
    assert calls == [(name, 1, 77) for name in NAMES]
    assert torch.cuda.current_device() == 0


def test_streams_of_another_gpu_are_refused(calls):
    with pytest.raises(ValueError, match="stream is of cuda:0"):
        three_calls(Stream(HERE, 5))
    assert calls == []


def test_capturing_is_looked_for_on_the_caches_gpu(calls, monkeypatch):
    from paper_2607_01308_amd import serving
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing",
                        lambda: torch.cuda.current_device() == 1)
    sc = object.__new__(serving.ServingCache)
    sc._held = on_gpu(2, dtype=torch.int32)
    for stream in (None, Stream(THERE, 5)):
        with pytest.raises(RuntimeError, match="captured"):
            sc._refuse_capture("extend", stream)
