"""The alternatives of rows with NaN (gmc_token_scores): a NaN is larger than all else, several
come by their place, and every place is one of the vocabulary's, the first and the last
included.  Whole numbers: compared with the 64-bit statement's, exactly."""
import math

import numpy as np
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# rows of one wavefront, of one workgroup, and cut in pieces (16 bits from 106,496 entries on, 32 from 53,248)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 4, 30, 300, 3000, 20000, 70000, 120001])
def test_nan_in_any_place(V, dtype):
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(V)
    x = torch.randn(9, 1, V, device="cuda:0", generator=g).to(dtype)
    x[0, 0, 0] = math.nan
    x[1, 0, 0], x[1, 0, V - 1] = -math.nan, math.nan
    x[2] = math.nan
    x[3, 0, V // 2] = math.inf
    x[3, 0, 0] = math.nan
    x[4], x[4, 0, 0] = -math.inf, math.nan
    x[5, 0, ::2] = math.nan
    x[6, 0, V - 1] = math.nan
    x[7, 0, :V // 2 + 1] = math.nan
    for top in sorted({1, min(V, 3), min(V, 32)}):
        _, entropy, top_logp, ids, norm = gmc.token_scores(x, top=top)
        assert np.array_equal(ids.cpu().numpy()[:, 0], ref.scores(x[:, 0].double().cpu().numpy(), 1.0, top)[3]), top
        assert torch.isnan(top_logp[:8]).all() and torch.isnan(entropy[:8]).all() and torch.isnan(norm[:8, :, 0]).all()
        assert torch.isfinite(top_logp[8]).all() and torch.isfinite(entropy[8]).all()
