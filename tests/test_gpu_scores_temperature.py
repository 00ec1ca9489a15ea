"""Logits of -inf at temperatures whose reciprocal is nothing, or nearly, in 32 bits: they still have no
probability, and all others the same."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("tau", [1e30, 1e40, 1e44, 1e46, 1e300])
@pytest.mark.parametrize("V", [5, 3000, 70000])
def test_masked_logits_at_high_temperatures(V, tau):
    import paper_1905_12948_amd as gmc
    x = torch.randn(1, 2, V, device="cuda:0")
    x[..., 3:] = -math.inf
    labels = torch.tensor([[V - 1, 1]], device="cuda:0")
    logp, entropy, top_logp, ids, norm = gmc.token_scores(x, labels, top=5, temperature=tau)
    # z is 0 to 2^-60 and what is left is ln 3: off by up to two units in its last place (2^-23), rounded once more
    near = 5 * 2.0 ** -24
    assert logp[0, 0] == -math.inf and abs(logp[0, 1].item() + math.log(3)) <= near
    assert (entropy - math.log(3)).abs().max() <= near
    assert (top_logp[..., 3:] == -math.inf).all() and (top_logp[..., :3] + math.log(3)).abs().max() <= near
    assert (ids[..., :3].sort(-1).values == torch.arange(3, device="cuda:0")).all()
    assert (ids[..., 3:] == torch.tensor([3, 4], device="cuda:0")).all()
