"""Numbers that the library takes in 32 bits: what does not fit is refused, never cut. On the CPU, with
stand-ins for the tensors' places on a GPU and for the library."""

import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2607_01308_amd import _cabi as C
from paper_2607_01308_amd import drafting, qcache

FAR = (2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 31 - 1, -2 ** 32)
i32 = torch.int32


class Seen(Exception):
    """The call reached the library."""


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Seen(name)
        return call


class OnGpu(torch.Tensor):
    """A CPU tensor that says it lives on a GPU."""
    is_cuda = True


@pytest.fixture
def cache(monkeypatch):
    stream = SimpleNamespace(cuda_stream=0, device=torch.device("cpu"))
    for module in (qcache, drafting):
        monkeypatch.setattr(module, "_use", lambda *a: (stream, True))
        monkeypatch.setattr(module, "_call", lambda here, device, f, *args: f(*args))
    monkeypatch.setattr(C, "lib", lambda: Library())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return SimpleNamespace(device=torch.device("cpu"), L=2, H=2, d=64, B=16, P=10,
                           codes=None, scales=None, struct=C.CmQcache(2, 2, 64, 16, 10, 256, 256))


def calls(cache):
    q, table, lens = torch.zeros((2, 4, 64)), torch.zeros((2, 3), dtype=i32), torch.zeros(2, dtype=i32)
    rows, pos = torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    kv, slots = torch.zeros((2, 2, 64)), torch.zeros(2, dtype=torch.int64)
    one = torch.zeros((2, 1), dtype=torch.int64)
    gpu = [x.as_subclass(OnGpu) for x in (pos, rows, lens)]

    def tree(window=0):
        return drafting.QCacheTree(one, pos, window)

    return {
        "write layer": lambda x: qcache.qcache_write(cache, x, kv, kv, slots),
        "attention layer": lambda x: qcache.qcache_attention(cache, x, q, table, lens),
        "attention window": lambda x: qcache.qcache_attention(cache, 0, q, table, lens, window=x),
        "attention max_rows": lambda x: qcache.qcache_attention(cache, 0, q, table, lens, rows, max_rows=x),
        "tree attention layer": lambda x: drafting.qcache_tree_attention(cache, x, q, table, lens, rows, tree()),
        "tree attention window": lambda x: drafting.qcache_tree_attention(cache, 0, q, table, lens, rows, tree(x)),
        "tree attention max_rows": lambda x: drafting.qcache_tree_attention(cache, 0, q, table, lens, rows, tree(),
                                                                            max_rows=x),
        "tree window": lambda x: drafting.qcache_tree(gpu[0], gpu[1], gpu[2], 2, 2, x),
        "copy layer": lambda x: drafting.qcache_copy(cache, pos, pos, x, 1),
        "copy layers": lambda x: drafting.qcache_copy(cache, pos, pos, 0, x),
        "tables block": lambda x: qcache.qcache_tables(10, x, lens, lens, pos, table, 2),
    }


@pytest.mark.parametrize("name", list(calls(None)))
def test_what_does_not_fit_is_refused(cache, name):
    call = calls(cache)[name]
    for x in FAR:
        with pytest.raises(ValueError, match=name.split()[-1]):
            call(x)
    for x in (0, 1, 2 ** 31 - 1, -1, -2 ** 31):              # (what is no layer or window the library refuses)
        with pytest.raises(Seen):
            call(x)


def test_ctypes_cuts():
    """Why: a number of more bits loses them without an error."""
    assert ctypes.c_int32(2 ** 32 + 5).value == 5 and C.CmQattention(window=2 ** 31).window == -2 ** 31
