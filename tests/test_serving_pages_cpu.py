"""Which pages belong to which sequence: the host bookkeeping of the paged cache (no GPU)."""
import pytest

from paper_2309_17224_b200 import build as B

B.build()
from paper_2309_17224_b200.serving import PagePool


def test_sequences_grow_page_by_page_and_give_them_back():
    pool = PagePool(6, 16)
    pool.extend(["a", "b"], [16, 1])
    assert pool.free_pages == 4 and pool.length("a") == 16
    pool.extend(["a"], [1])
    pool.extend(["b"], [15])
    assert pool.free_pages == 3
    start, lens, rows = pool.indices(["b", "a"], [15, 1])
    assert start == [0, 15, 16] and lens == [16, 17]
    assert len(rows[0]) == 2 and len({rows[0][0], *rows[1]}) == 3       # nobody shares a page
    taken = set(rows[1])
    pool.release("a")
    assert pool.free_pages == 5 and pool.length("a") == 0
    pool.extend(["c"], [33])
    assert taken <= set(pool.indices(["c"], [33])[2][0])


def test_a_call_that_does_not_fit_changes_nothing():
    pool = PagePool(3, 32)
    pool.extend([1], [40])
    with pytest.raises(MemoryError):
        pool.extend([1, 2], [30, 33])
    assert pool.length(1) == 40 and pool.length(2) == 0 and pool.free_pages == 1
    pool.extend([2], [0])
    assert pool.indices([2], [0]) == ([0, 0], [0], [[0]])


def test_bad_arguments():
    with pytest.raises(ValueError):
        PagePool(4, 48)
    pool = PagePool(4, 16)
    for seqs, new in ((["a", "a"], [1, 1]), (["a"], [1, 2]), (["a"], [-1])):
        with pytest.raises(ValueError):
            pool.extend(seqs, new)
