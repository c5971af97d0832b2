"""Pins of the oracle's pages (oracle/kv_stream_oracle.py) where a pool runs dry, by hand."""
from oracle import kv_stream_oracle as W


def test_an_entry_whose_first_tokens_were_lost_stays_without_a_page():
    p = W.Pages(2, 32)
    a, b = [[-1] * 3], [[-1] * 3]
    assert p.reserve(a, [64], [64]) == ([(-1, -1, 0)], 0)
    assert p.reserve(b, [5], [5]) == ([(-1, -1, 0)], 1) and b == [[-1] * 3]
    p.release(a)
    assert p.reserve(b, [1], [6]) == ([(-1, -1, 0)], 1) and b == [[-1] * 3] and p.refs == [0, 0]      # tokens 0 to 4 are nowhere
    assert p.reserve(b, [30], [36]) == ([(-1, -1, 0)], 1) and b == [[-1, 0, -1]] and p.refs == [1, 0]
    assert p.reserve(b, [28], [64]) == ([(-1, -1, 0)], 0) and b == [[-1, 0, -1]]
    assert p.reserve(b, [1], [65]) == ([(-1, -1, 0)], 0) and b == [[-1, 0, 1]]


def test_what_names_no_page_is_left_as_it_is():
    p = W.Pages(3, 32)
    t = [[7, 9, -5]]
    assert p.reserve(t, [40], [50]) == ([(-1, -1, 0)], 1) and t == [[7, 0, -5]]      # tokens 10 to 49 behind ten that are nowhere
    assert p.reserve(t, [32], [96]) == ([(-1, -1, 0)], 0) and t == [[7, 0, 1]] and p.refs == [1, 1, 0]


def test_a_call_that_is_repeated():
    p = W.Pages(2, 32)
    t = [[-1] * 2, [-1] * 2]
    assert p.reserve(t, [40, 20], [40, 20])[1] == 1 and t == [[0, 1], [-1, -1]]
    p.release(t, [32, 0])
    assert p.reserve(t, [0, 20], [32, 20])[1] == 0 and t == [[0, -1], [1, -1]]


def test_the_last_holders_of_a_page_leave_it_to_the_first_of_them():
    p = W.Pages(3, 32)
    t, c, lens = [[-1] * 2], [[-1] * 2 for _ in range(3)], [0] * 3
    p.reserve(t, [20], [20])
    p.fork(t, [20], [0, 0, 0], c, lens)
    assert p.refs == [4, 0, 0]
    p.release(t)
    assert p.reserve(c, [0, 1, 1], [20, 21, 21]) == ([(-1, -1, 0), (0, 1, 20), (0, 2, 20)], 0) and p.refs == [1, 1, 1]      # (the first one stands still)
    p.release(c, [0, 0, 64])
    d, lens = [[-1] * 2 for _ in range(3)], [0] * 3
    p.fork(c, [0, 0, 21], [2, 2, 2], d, lens)
    p.release(c)
    assert p.refs == [0, 0, 3]
    assert p.reserve(d, [1, 1, 20], [22, 22, 41]) == ([(-1, -1, 0), (2, 0, 21), (2, 1, 21)], 1) and d == [[2, -1], [0, -1], [1, -1]] and p.refs == [1, 1, 1]


def test_a_holder_that_is_not_there_keeps_the_page_shared():
    p = W.Pages(4, 32)
    p.refs = [3, 0, 0, 0]
    assert p.reserve([[0, -1], [0, -1]], [1, 1], [5, 9]) == ([(0, 1, 4), (0, 2, 8)], 0) and p.refs == [1, 1, 1, 0]
    p.refs = [2, 0, 0, 0]
    t = [[-1, 0], [0, -1]]      # at other places: as of any page with a count above one
    assert p.reserve(t, [1, 1], [33, 1]) == ([(-1, -1, 0)] * 2, 0) and t == [[-1, 1], [2, -1]] and p.refs == [0, 1, 1, 0]
