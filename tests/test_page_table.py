"""The host's table of a paged cache: pages are handed out for all sequences of a step or for none."""
import pytest

from paper_2609_19758_b200.attention_layer import PageTable


def state(t):
    return (sorted(t.free), [list(r) for r in t.rows], list(t.length))


def test_pages_follow_the_lengths():
    t = PageTable(6, 4)
    a, b = t.open(), t.open()
    t.extend(a, 5)
    t.extend(b, 4)
    assert [len(r) for r in t.rows] == [2, 1] and t.length == [5, 4] and len(t.free) == 3
    t.extend(a, 0)
    t.extend(a, 3)
    assert [len(r) for r in t.rows] == [2, 1] and t.length == [8, 4]
    assert len({p for r in t.rows for p in r} | set(t.free)) == 6
    t.close(a)
    assert len(t.free) == 5 and t.length == [0, 4]


def test_a_full_cache_leaves_the_table_as_it_was():
    t = PageTable(3, 4)
    a, b = t.open(), t.open()
    t.extend(a, 6)
    before = state(t)
    with pytest.raises(RuntimeError, match="full"):
        t.extend(a, 7)                       # two pages more, one is free
    assert state(t) == before
    with pytest.raises(RuntimeError, match="full"):
        t.extend_all([b, a], [4, 4])         # each alone would fit
    assert state(t) == before
    t.extend_all([b, a], [4, 2])
    assert t.length == [8, 4] and not t.free


@pytest.mark.parametrize("seqs,tokens", [([0, 0], [1, 1]), ([0], [1, 2]), ([0, 1], [1, -1]), ([2], [1]), ([-1], [1])])
def test_sequences_that_make_no_step(seqs, tokens):
    t = PageTable(8, 4)
    t.open(), t.open()
    before = state(t)
    with pytest.raises(ValueError):
        t.extend_all(seqs, tokens)
    assert state(t) == before


def test_tokens_are_taken_back():
    t = PageTable(6, 4)
    a, b = t.open(), t.open()
    t.extend_all([a, b], [6, 1])
    before = state(t)
    t.extend_all([a, b], [7, 3])
    t.retract([a, b], [7, 3])
    assert state(t) == before
    t.retract([a], [6])
    assert t.length == [0, 1] and not t.rows[a]
    for seqs, tokens in (([b], [2]), ([a], [1]), ([b], [-1]), ([b, b], [1, 1]), ([5], [0])):
        with pytest.raises(ValueError):
            t.retract(seqs, tokens)
    assert t.length == [0, 1]
