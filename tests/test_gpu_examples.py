"""examples/train_workers.py on the GPU: the operators of a worker's pass and GMC's
iteration together lower the preference loss and raise the rollouts' reward."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_train_workers():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import train_workers
    finally:
        sys.path.pop(0)
    said = []
    first, last, right0, right1 = train_workers.train(30, 60, log=said.append)
    print("\n".join(said), flush=True)
    assert abs(first - 0.6931) < 0.01       # the model is its own reference: log 2, dropout aside
    assert last < 0.2 * first
    assert right1 > 1.3 * right0
