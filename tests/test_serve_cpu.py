"""Page accounting of serve.py."""
import numpy as np
import pytest

from paper_2607_21291_gb300.serve import PagePool


def test_pages_are_taken_as_needed_and_given_back():
    p = PagePool(10, 16, 2, 2, 4)
    assert not p.reserve(np.zeros((2, 2), dtype=np.int64))
    assert p.reserve(np.array([[16, 17], [0, 1]]))
    assert p.held.tolist() == [[1, 2], [0, 1]] and len(p.free) == 6
    assert not p.reserve(np.array([[16, 32], [0, 16]]))
    assert not p.reserve(np.array([[1, 1], [0, 0]])) and p.held[0, 1] == 2   # what is held stays
    used = [int(x) for l in range(2) for b in range(2) for x in p.table[l, b, :p.held[l, b]]]
    assert len(set(used)) == 4 and not set(used) & set(p.free)
    p.release(1)
    assert p.held.tolist() == [[1, 0], [0, 0]] and len(p.free) == 9 and len(set(p.free)) == 9


def test_a_refusal_takes_nothing():
    p = PagePool(3, 16, 1, 2, 4)
    p.reserve(np.array([[16, 0]]))
    with pytest.raises(MemoryError):
        p.reserve(np.array([[32, 32]]))
    with pytest.raises(ValueError):
        p.reserve(np.array([[65, 0]]))
    assert p.held.tolist() == [[1, 0]] and len(p.free) == 2
