"""The attention block of examples/: quantized layers, append, attention and gather together, in ragged chunks and in a captured graph."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int4", "fp4", "w8a8"])
def test_attention_block(fmt):
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "attention_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    held, whole = m.main(tokens=30, fmt=fmt, verbose=False)
    # f16 weights and a bf16 output: 2^-9 each in the mean, within 2^-7.  Codes of three mantissa bits: an error uniform in half a step is 2^-4 / sqrt(3) of
    # a number's power of two at most, 0.036, in values that weights then average, and in keys (scores off by 0.036 |q| |k| / sqrt(DIM) / sqrt(DIM) of a product of
    # about 3 x 3, hence 0.04 of a weight): within 0.08 together.
    assert held <= 2.0 ** -7 and whole <= 0.08
