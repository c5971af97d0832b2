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
