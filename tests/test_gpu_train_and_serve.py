"""The vocabulary head's operators together, as examples/train_and_serve.py uses them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_head_learns_and_is_served_from_four_bits():
    spec = importlib.util.spec_from_file_location("train_and_serve", os.path.join(ROOT, "examples", "train_and_serve.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, served, off = example.run(rounds=40, prompts=256, vocab=2003, width=256)
    # a tenth of the tokens is favoured: chance gives 0.1, with a standard deviation of 0.02 over 256 prompts
    assert first < 0.2 and last > 0.4 and served > 0.4 and off < 2.0
