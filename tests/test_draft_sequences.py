"""Which tokens and pages the sequences of a decoder block hold while drafts wait: the bookkeeping alone, without a GPU."""
import pytest

from paper_2511_00603_amd import binding as B
from paper_2511_00603_amd.decoder import DecoderBlock
from test_decoder_sequences import X, block, refused, state, taken


def drafted(b, new, parents):
    b._commit(b._admit(new), b._trees(new, parents))


def test_drafts_hold_their_pages_but_are_no_tokens_yet():
    b = block()
    b.device = "cpu"
    taken(b, [[("a", X(60))], [("b", X(3))]])
    drafted(b, [[("a", X(10))], []], [{"a": [-1] + [0] * 9}, None])
    assert b.sequences[0]["a"][1] == 60 and len(b.sequences[0]["a"][0]) == 2 and b.drafts[0]["a"] == (60, [-1] + [0] * 9) and not b.drafts[1]
    refused(b, [[("a", X(1))], []], ValueError)                  # it waits
    with pytest.raises(ValueError):
        b.fork(0, "a", "a2")
    taken(b, [[], [("b", X(1))]])                                # others go on
    for bad in ([None, {}], [None], [{"logits": X(3)}, None]):
        with pytest.raises(ValueError):
            b.accept(bad, [[1.0], []])
    before = state(b)
    assert before[0][0]["a"][1] == 60
    b.release(0, "a")
    assert b.pools[0].n_free == 6 and not b.drafts[0]


@pytest.mark.parametrize("parents", [[{"a": [0]}, None], [{"a": [-1, 0, 1]}, None], [{"x": [-1]}, None], [{"a": []}, None], [None]])
def test_parents_that_do_not_fit_are_refused(parents, monkeypatch):
    b = block()
    taken(b, [[("a", X(5))], []])
    before = state(b)
    with pytest.raises(ValueError):
        b.step([[("a", X(2))], []], parents)
    assert state(b) == before and not any(b.drafts)
    b = block(n_pages=9)
    with pytest.raises(ValueError):                              # more rows than a tree may have
        b.step([[("a", X(B.EPARA_TREE_MAX_ROWS + 1))], []], [{"a": list(range(-1, B.EPARA_TREE_MAX_ROWS))}, None])


def test_a_step_of_drafts_that_fails_leaves_nothing_waiting(monkeypatch):
    b = block()
    taken(b, [[("a", X(60))], []])
    before = state(b)

    def broken(*_):
        raise RuntimeError("no memory")

    monkeypatch.setattr(DecoderBlock, "_launch", broken)
    with pytest.raises(RuntimeError):
        b.step([[("a", X(8))], []], [{"a": list(range(-1, 7))}, None])
    assert state(b) == before and not any(b.drafts)
