"""The example of an attention block runs: the gate passes the ways that are right and no others."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attention_block():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    passed = example.main(["--requests", "5", "--tokens", "300", "--heads", "8", "--kv-heads", "2", "--dim", "64", "--repeats", "3"])
    assert passed["the library"] and passed["plain, 32 bits"]
    assert not passed["wrong scale"] and not passed["sees the next token"]
