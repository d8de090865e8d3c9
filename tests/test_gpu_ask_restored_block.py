"""Append and attention around save and restore: the example's path, in both cache types."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("block,question", [(333, 21), (16, 1), (129, 200)])
def test_a_restored_block_answers_with_the_same_bits(fp8, block, question):
    spec = importlib.util.spec_from_file_location("ask_restored_block", os.path.join(ROOT, "examples", "ask_restored_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(fp8, block, question) == 0
