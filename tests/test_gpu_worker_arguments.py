"""Arguments the binding refuses that the C interface could not see: whole numbers
beyond its integers, of which it would get the low bits."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_integers_beyond_the_interface():
    import paper_1905_12948_amd as gmc
    x = torch.zeros(2, 3, 8, device="cuda:0")
    for more in (dict(site=2 ** 32), dict(site=2 ** 31), dict(worker=2 ** 32 + 1), dict(t=2 ** 64), dict(t=2 ** 63)):
        with pytest.raises(ValueError, match="integer"):
            gmc.dropout(x, 0.1, 1, **more)
        with pytest.raises(ValueError, match="integer"):
            gmc.dropout_backward(x, 0.1, 1, **more)
    with pytest.raises(gmc.GmcError):
        gmc.dropout(x, 0.1, 1, worker=64)
    with pytest.raises(ValueError, match="integer"):
        gmc.group_norm(x, 2 ** 32 + 2)
    labels = torch.zeros(2, 3, device="cuda:0", dtype=torch.int64)
    with pytest.raises(ValueError, match="integer"):
        gmc.policy_loss(x, labels, None, torch.ones(2, device="cuda:0"), ignore=2 ** 64)
    with pytest.raises(ValueError, match="integer"):
        gmc.preference_loss(x, labels, ignore=2 ** 64)


def test_channels_beyond_the_interface():
    import paper_1905_12948_amd as gmc
    x = torch.empty(1, 2 ** 32 + 8, device="cuda:0", dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="integer"):
        gmc.group_norm(x, 2)
    one = torch.zeros(1, 2, device="cuda:0")
    with pytest.raises(ValueError, match="integer"):
        gmc.group_norm_backward(x, x, one, one)
