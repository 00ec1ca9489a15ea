"""Matrices whose norm is far below eps (gmc_orthogonalize): down to |M| / (|M| + eps) = 2^-126, the smallest normal
number of 32 bits, results are as exact as others'.

One step that leaves X as it is (1, 0, 0): a kept value is off by 2^-22 of it (entries are above 2^-27 of |M|), the
polynomial is the identity, and theta, alpha scale theta, its product with an entry and the result round once each,
2^-24; a kept X is off by 2^-24 before it is split: 2^-22 + 5 * 2^-24 < 2^-21, entry by entry, and 2^-149."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# one workgroup's, many workgroups', on its side
@pytest.mark.parametrize("rows,cols", [(50, 60), (200, 210), (210, 140)])
@pytest.mark.parametrize("alpha", [1.0, 2.0 ** 90])
@pytest.mark.parametrize("size,eps", [(1.7 * 2.0 ** -126, 1.0), (1.3 * 2.0 ** -119, 1.0), (1.7 * 2.0 ** -118, 1.0), (1.4 * 2.0 ** -114, 0.5),
                                      (1.7 * 2.0 ** -100, 1.0), (1.7 * 2.0 ** -20, 1.0)])
def test_far_below_eps(rows, cols, size, eps, alpha):
    import paper_1905_12948_amd as gmc
    m = np.random.default_rng(rows).uniform(0.5, 1.0, (rows, cols))
    x = torch.as_tensor(m / np.linalg.norm(m) * size, dtype=torch.float32).cuda()
    exact = x.double().cpu().numpy()
    norm = np.linalg.norm(exact)
    assert norm / (norm + eps) >= 2.0 ** -126
    plan = gmc.Matrices(rows * cols, [(0, rows, cols)])
    got = gmc.orthogonalize(plan, x.reshape(-1), eps=eps, alpha=alpha, steps=1, coefficients=(1.0, 0.0, 0.0)).view(rows, cols).double().cpu().numpy()
    want = alpha * exact / (norm + eps)
    assert (np.abs(got - want) <= 2.0 ** -21 * np.abs(want) + 2.0 ** -149).all(), np.abs(got / want - 1).max()
