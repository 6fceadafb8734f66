"""The calls together, as the example runs them: tree decoding gives the tokens of plain decoding."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("hybrid_decode", os.path.join(ROOT, "examples", "hybrid_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_trees_decode_what_single_tokens_do(example, capsys):
    """fp32: the two orders of summation differ in the last bits of a logit (1e-6), a drawn point lies that near a boundary once
    in some 1e4 tokens, and here are 192."""
    plain, tree, steps, rounds = example.main(["--tokens", "48"])
    assert plain == tree and steps == 48 and rounds < steps
    assert "192 of 192 tokens agree" in capsys.readouterr().out


def test_bf16_runs(example):
    plain, tree, _, rounds = example.main(["--tokens", "16", "--sequences", "2", "--dtype", "bf16"])
    assert all(len(t) == 16 for t in plain + tree) and rounds <= 16
    assert all(p[0] == t[0] for p, t in zip(plain, tree))              # the first token is given
