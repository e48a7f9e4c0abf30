"""Steps of ServingCache that fail leave nothing changed, and steps that cannot be are refused before anything
is, on the CPU with the plain stand-ins of test_serving_drafts.py."""

import pytest
import torch

from paper_2607_01308_amd import serving
from test_serving import plain  # noqa: F401
from test_serving_drafts import cache_of, check, numbers  # noqa: F401


def state(sc):
    return list(sc.lengths), sc.free_pages, sc._held.tolist(), [list(x) for x in sc._shared]


def grown(sc):
    """Place 0 with 20 tokens, which the stand-in's pages hold."""
    step = sc.extend([20] + [0] * (sc.places - 1))
    for i, slot in enumerate(step.tables.slots.tolist()):
        sc.cache.tokens[slot // sc.cache.B, slot % sc.cache.B] = i
    return [list(range(20))] + [[] for _ in range(sc.places - 1)]


@pytest.mark.parametrize("part", ["qcache_tree", "upload"])
def test_a_draft_that_fails_changes_nothing(numbers, monkeypatch, part):  # noqa: F811
    sc = cache_of(10, 16, 2, 100)
    want = grown(sc)
    before = state(sc)

    def refuse(*args, **kwargs):
        raise RuntimeError("refused")

    with monkeypatch.context() as m:
        if part == "upload":
            m.setattr(sc, "_upload", refuse)
        else:
            m.setattr(serving, "qcache_tree", refuse)
        for _ in range(3):
            with pytest.raises(RuntimeError, match="refused"):
                sc.draft([[-1] + [0] * 20, [-1]])
            assert state(sc) == before
    check(sc, want)
    step = sc.draft([[-1, 0], []])
    assert sc.lengths == [22, 0] and step.tokens == 2


@pytest.mark.parametrize("window", [-1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63])
def test_windows_of_no_32_bits(numbers, window):  # noqa: F811
    sc = cache_of(10, 16, 2, 100)
    grown(sc)
    before = state(sc)
    with pytest.raises(ValueError, match="window"):
        sc.draft([[-1, 0], []], window=window)
    assert state(sc) == before
    sc.draft([[-1, 0], []], window=2 ** 31 - 1)


def test_counts_and_parents_that_are_no_numbers(numbers):  # noqa: F811
    sc = cache_of(10, 16, 2, 100)
    grown(sc)
    before = state(sc)
    with pytest.raises((TypeError, ValueError)):
        sc.draft([["a"], []])
    assert state(sc) == before
    step = sc.draft([[-1, 0], []])
    after = state(sc)
    with pytest.raises((TypeError, ValueError)):
        sc.accept(step, torch.zeros(2, dtype=torch.int32), [None, 0])
    assert state(sc) == after


def test_accept_tells_what_became_of_the_path(numbers, monkeypatch):  # noqa: F811
    """The status that the library leaves on the device is the caller's to ask for."""
    from paper_2607_01308_amd._cabi import CmError
    from paper_2607_01308_amd.drafting import QCacheKept

    sc = cache_of(10, 16, 2, 100)
    grown(sc)
    step = sc.draft([[-1, 0, 0], [-1]])
    kept = sc.accept(step, torch.tensor([0, 2, -1, 0], dtype=torch.int32), [2, 1])
    assert kept.check() is kept and kept.lens.tolist() == sc.lengths == [22, 1]
    assert kept.info.tolist() == [0, 0]

    bad = QCacheKept(torch.zeros(2, dtype=torch.int32), torch.tensor([2, 0]))
    step = sc.draft([[-1, 0, 0], []])
    monkeypatch.setattr(serving, "qcache_keep", lambda *a, **k: bad)
    with pytest.raises(CmError, match="path"):
        sc.accept(step, torch.tensor([0, 2, 1], dtype=torch.int32), [3, 0]).check()


class Failing:
    """torch functions that fail from the n-th call on."""
    def __init__(self, real, after):
        self.real, self.left = real, after

    def __call__(self, *args, **kwargs):
        self.left -= 1
        if self.left < 0:
            raise RuntimeError("out of memory")
        return self.real(*args, **kwargs)


@pytest.mark.parametrize("what", ["release", "fork", "accept", "extend"])
@pytest.mark.parametrize("after", [0, 1, 2])
def test_steps_without_memory_change_nothing(numbers, monkeypatch, what, after):  # noqa: F811
    """Whatever allocation of a step fails: lengths, pages and who shares them are as before, and the step can
    be taken again."""
    sc = cache_of(14, 16, 3, 100)
    want = grown(sc)
    sc.fork(0, 1)
    want[1] = list(want[0])
    step = sc.draft([[-1, 0, 1] + [0] * 20, [], []])
    ids = [100 + i for i in range(23)]
    for slot, x in zip(step.tables.slots.tolist(), ids):
        sc.cache.tokens[slot // 16, slot % 16] = x
    if what != "accept":
        sc.accept(step, torch.tensor([0, 1, 2] + [-1] * 20, dtype=torch.int32), [3, 0, 0])
        want[0] = want[0] + ids[:3]
        # (the buffer of free pages is to be moved to its front by the next release)
        for _ in range(3):
            sc.extend([0, 0, 60])
            sc.release(2)
    calls = {"release": lambda: sc.release(0), "fork": lambda: sc.fork(0, 2), "extend": lambda: sc.extend([5, 0, 2]),
             "accept": lambda: sc.accept(step, torch.tensor([0, 1, 2] + [-1] * 20, dtype=torch.int32), [3, 0, 0])}
    before, runs = state(sc), [[(run.pages, run.places) for run in x] for x in sc._shared]
    failed = False
    with monkeypatch.context() as m:
        # (clones of tensors, and tensors from the host)
        clone, made = Failing(torch.Tensor.clone, after), Failing(torch.tensor, after)
        m.setattr(torch.Tensor, "clone", lambda t: clone(t))
        m.setattr(torch, "tensor", made)
        try:
            calls[what]()
        except RuntimeError:
            failed = True
    if not failed:
        return
    assert state(sc) == before and [[(run.pages, run.places) for run in x] for x in sc._shared] == runs
    if what in ("release", "fork"):
        check(sc, want)
        calls[what]()
        if what == "release":
            want[0] = []
        else:
            want[2] = list(want[0])
        check(sc, want)
