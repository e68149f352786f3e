"""The page bookkeeping of the answering stacks and where they take their weights from (CPU only)."""
import pytest

from paper_2406_14898_gb300.generate import BlockStack, Pages


def state(p):
    return list(p.lens), [list(h) for h in p.held], list(p.free), p.table.tolist()


@pytest.mark.parametrize("n_pages,lens,new,error", [
    (3, [5, 30], [3, 20], MemoryError),        # sequence 1 finds no page
    (3, [5, 16], [12, 17], MemoryError),       # each alone would find one, both do not
    (9, [5, 30], [3, 35], ValueError),         # sequence 1 is too long
    (9, [5, 30, 0], [20, 1, 65], ValueError),
])
def test_a_refused_extension_changes_nothing(n_pages, lens, new, error):
    p = Pages(n_pages, 16, len(lens), 64)
    p.extend(lens)
    before = state(p)
    with pytest.raises(error):
        p.extend(new)
    assert state(p) == before


def test_pages_are_handed_out_and_come_back():
    p = Pages(6, 16, 2, 64)
    p.extend([17, 3])
    assert p.lens == [17, 3] and [len(h) for h in p.held] == [2, 1] and len(p.free) == 3
    assert p.table[0, :2].tolist() == p.held[0] and p.table[1, 0] == p.held[1][0]
    assert len(set(p.held[0] + p.held[1] + p.free)) == 6
    p.extend([15, 13])
    assert [len(h) for h in p.held] == [2, 1]
    p.drop(0)
    assert p.lens == [0, 16] and p.table[0].tolist() == [-1] * 4 and len(p.free) == 5
    p.extend([64, 0])
    assert p.lens == [64, 16]


@pytest.mark.parametrize("lens,new", [([5, 30], [3, 20]), ([16, 0, 7], [0, 33, 9]), ([0, 0], [16, 1])])
def test_an_extension_is_taken_back(lens, new):
    p = Pages(9, 16, len(lens), 64)
    p.extend(lens)
    before = state(p)
    p.extend(new)
    p.shorten(new)
    assert state(p) == before
