"""The command line of examples/train_workers.py gives train its arguments (no GPU)."""
import inspect
import os
import sys

import pytest

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import train_workers
    finally:
        sys.path.pop(0)
    return train_workers


@pytest.mark.parametrize("line,want", [([], (False, 0.0)), (["--orthogonal"], (True, 0.0)), (["--bonus", "0.02"], (False, 0.02)),
                                       (["--bonus=0.02", "--orthogonal"], (True, 0.02))])
def test_options(example, line, want):
    got = example.options(line)
    assert (got["orthogonal"], got["bonus"]) == want
    assert set(got) <= set(inspect.signature(example.train).parameters)
