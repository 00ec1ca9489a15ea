"""A plan that is dropped while a stream is captured does not end the capture, and calls in the graph go
on with theirs."""
import gc

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_dropped_during_a_capture():
    import paper_1905_12948_amd as gmc
    from paper_1905_12948_amd import matrix
    n = 100 * 90
    x = torch.randn(n, device="cuda:0")
    kept, closed, dropped = (gmc.Matrices(n, [(0, 100, 90)]) for _ in range(3))
    want = gmc.orthogonalize(kept, x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        closed.close()
        del dropped
        gc.collect()
        out = gmc.orthogonalize(kept, x)
    assert len(matrix._dropped) == 2
    for k in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        if k == 0:
            gmc.Matrices(n, [(0, 9, 9)]).close()
            assert not matrix._dropped
