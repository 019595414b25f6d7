"""The pages' oracle against hand-worked cases (CPU)."""
import numpy as np

from oracle.pages import Book


def test_by_hand():
    b = Book(np.zeros(6), np.zeros((4, 3)), np.zeros(4), 4)
    assert b.grow([5, 1], T=7) == ([5, 1], [0, 1, 2, 3, 4, 8, -1], [0, 1, 2, 3, 4, 0, 0])
    assert b.held() == [[0, 1], [2], [], []] and b.refs.tolist() == [1, 1, 1, 0, 0, 0]
    assert b.fork([0, 1, 0], [2, 3, 2]) == ([5, 1, -1], [1, 2, -1], [3, 4, -1])
    assert b.held() == [[0, 1], [2], [0, 3], [4]] and b.refs.tolist() == [2, 1, 1, 1, 1, 0]
    b.check()
    assert b.grow([4, 4, 0], [3, 1, 0])[0] == [5, -1, 5]  # one page is left
    b.free([0, 0])
    assert b.refs.tolist() == [1, 0, 1, 1, 1, 1] and b.held()[0] == []
    assert b.compact(3) == ([5, -1, -1], [1, -1, -1])
    assert b.held() == [[], [2], [0, 3], [4, 1]] and b.refs.tolist() == [1, 1, 1, 1, 1, 0]
    b.check()
