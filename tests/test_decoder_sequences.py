"""Which tokens and pages the sequences of a decoder block hold after steps that are refused: the bookkeeping alone, without a GPU."""
import copy
from types import SimpleNamespace

import pytest
import torch

from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd import runtime as R
from paper_2511_00603_amd.decoder import DecoderBlock


def block(n_pages=6, services=2, d=16, max_tokens=300):
    b = DecoderBlock.__new__(DecoderBlock)
    b.params = [SimpleNamespace(Wqkv=torch.zeros(d, 8)) for _ in range(services)]
    b.pools, b.sequences = [R.PagePool(n_pages) for _ in range(services)], [{} for _ in range(services)]
    b.rotary = torch.zeros(max_tokens, 4, 2)
    return b


def X(n, d=16):
    return torch.zeros(n, d, dtype=torch.bfloat16)


def state(b):
    return copy.deepcopy(b.sequences), [(p.n_free, p.refs.tolist(), p.free_pages[: p.n_free].tolist()) for p in b.pools]


def taken(b, new):
    """A step without its launches."""
    b._commit(b._admit(new))


def refused(b, new, error):
    before = state(b)
    with pytest.raises(error) as e:
        b.step(new)
    assert state(b) == before
    return e.value


def test_a_step_that_is_refused_changes_nothing():
    b = block()
    taken(b, [[("a", X(60))], [("b", X(130)), ("c", X(1))]])
    assert b.sequences[0]["a"][1] == 60 and [len(s[0]) for s in b.sequences[1].values()] == [3, 1]
    # the pool runs out at the second sequence, at a second service, and for a name that is not known yet
    for new in ([[], [("b", X(60)), ("c", X(200))]], [[("a", X(10))], [("c", X(230))]], [[("a", X(1))], [("new", X(150))]], [[("x", X(64)), ("y", X(64)), ("z", X(300))], []]):
        assert refused(b, new, B.EparaError).status == B.EPARA_ERR_CAPACITY
    # more positions than the table of angles has, a name twice, tokens of another width or type, another number of services
    for new in ([[("a", X(241))], []], [[("a", X(1))], [("b", X(1)), ("b", X(1))]], [[("a", X(1))], [("b", X(1, 24))]], [[("a", X(1).float())], []],
                [[("a", X(1)[0])], []], [[("a", X(1))]]):
        refused(b, new, ValueError)
    # and what fits afterwards goes on where it was
    b.release(1, "c")
    taken(b, [[("a", X(1))], [("b", X(1)), ("new", X(150))]])
    assert b.sequences[0]["a"][1] == 61 and b.sequences[1]["b"][1] == 131 and b.sequences[1]["new"][1] == 150


def test_pages_go_back_when_something_fails_after_they_were_taken(monkeypatch):
    """Whatever raises between the pages and the last launch: the sequences are what they were, and the pages are free in their old order."""
    b = block()
    taken(b, [[("a", X(60))], [("b", X(64))]])

    def broken(*_):
        raise RuntimeError("no memory")

    monkeypatch.setattr(DecoderBlock, "_launch", broken)
    refused(b, [[("a", X(70)), ("n", X(5))], [("b", X(100))]], RuntimeError)


def test_a_fork_or_a_compaction_whose_copy_fails_changes_nothing(monkeypatch):
    def broken(*_):
        raise RuntimeError("no memory")

    b = block(n_pages=10)
    b.device, b.caches = "cpu", [None, None]
    taken(b, [[("a", X(100)), ("b", X(64)), ("c", X(10))], []])
    b.release(0, "b")
    before = state(b)
    monkeypatch.setattr(R, "PageCopyPlan", broken)
    for f in (lambda: b.fork(0, "a", "child"), lambda: b.compact(0)):
        with pytest.raises(RuntimeError):
            f()
        assert state(b) == before
    with pytest.raises(ValueError):
        b.fork(0, "a", "c")                                      # a name that is taken
    assert state(b) == before
    monkeypatch.setattr(R, "PageCopyPlan", lambda groups, device: groups)
    copied = []
    monkeypatch.setattr(R, "copy_pages", copied.extend)
    b.fork(0, "a", "child")
    b.compact(0)
    assert [len(s[0]) for s in b.sequences[0].values()] == [2, 1, 2] and len(copied) == 1       # nothing lies above the pages in use: the child took the gap
