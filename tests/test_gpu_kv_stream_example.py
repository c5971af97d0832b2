"""The streaming attention block runs, in few pages, and its attention is that of the cache's own numbers."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,tokens", [("int4", 300), ("fp4", 3), ("w8a8", 70)])
def test_the_example_runs(fmt, tokens):
    from examples.stream_block import main
    error, used, pages = main(tokens, fmt, verbose=False)
    # the output's bf16 is off by 2^-8 of a number at most; normalised queries and weights in 16 bits of 2^-11 each move scores and weights by less than that again
    assert error <= 2.0 ** -7 and used <= pages
