"""gmc_orthogonal_step's (1 - decay) w + rate scale X: the decay takes its share however small
it is, the largest included.

Tolerances, with u = 2^-24.  One component, without a step: the result's rounding, that of decay
and of decay w (or of 1 - decay): u (2 |result| + 2 decay |w|).  The mean share that many
components lose, sum(w (w - result)) / sum(w^2): a rounding's error is at most u |result| with any sign, as
likely one as the other, so the mean of n of normal w is off by no more than u sqrt(3 / n) in the mean square
(the mean of w^4 is 3); six times that.

To the mean comes what is left where a decay takes few units in the last place.  For w between 2^k and 2^(k+1),
w = M ulp with ulp = 2^(k-23), the result loses round(y) units for y = decay M: an error of s(y) = round(y) - y units, a
sawtooth whose integral over any stretch is at most 1/8 (half a tooth's), and over a stretch with a weight that
rises and then falls at most 1/2 of the largest weight (the second mean value theorem, twice).  The
weight is 2 phi(w) w ulp with dw = ulp dy / decay, so the sum of w (w - result) is off by at most (1/2) 2^-46 / decay times
the sum over k of 4^k max(2 phi(w) w): 0.02 + 0.12 + 0.48 + 0.86 + 0.02 for k = -2 to 2 and less than 0.01 for the
others, 1.51.  Of the sum of w^2, which is 1 a component, that is below 2^-46 / decay."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# one workgroup's, many workgroups', and on its side
SHAPES = [(64, 70), (256, 300), (300, 256)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("decay", [1e-6, 3e-7, 1e-5, 0.003])
def test_mean_decay(rows, cols, decay):
    """No update and no momentum: X is 0."""
    import paper_1905_12948_amd as gmc
    n = rows * cols
    w = torch.randn(n, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(3))
    plan = gmc.Matrices(n, [(0, rows, cols)])
    out = gmc.orthogonal_step(plan, w, torch.zeros_like(w), None, 0.02, decay=decay, w_out=torch.empty_like(w))
    a, b = w.double(), out.double()
    share = ((a * (a - b)).sum() / (a * a).sum()).item()
    assert abs(share - decay) <= 6 * U * math.sqrt(3 / n) + 2.0 ** -46 / decay, (share, decay)


@pytest.mark.parametrize("decay", [1e-8, 2e-9])
def test_decays_below_a_rounding(decay):
    """Less than half a unit in w's last place: the step's own bits decide which components change, and
    as many do as the decay says (the difference of two results: twice the mean square)."""
    import paper_1905_12948_amd as gmc
    rows = cols = 2048
    n = rows * cols
    g = torch.Generator("cuda:0").manual_seed(4)
    w, u = (torch.randn(n, device="cuda:0", generator=g) for _ in range(2))
    plan = gmc.Matrices(n, [(0, rows, cols)])
    with_it, without = (gmc.orthogonal_step(plan, w, u, None, 0.02, decay=v, w_out=torch.empty_like(w)).double() for v in (decay, 0.0))
    a = w.double()
    share = ((a * (without - with_it)).sum() / (a * a).sum()).item()
    assert abs(share - decay) <= 6 * U * math.sqrt(2 * 3 / n), (share, decay)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("decay", [0.0, 1e-6, 0.01, 0.4999, 0.5, 0.5001, 0.7, 0.999999, 1.0, 1.5, 2.0, -0.01, -1.0])
def test_each_component(rows, cols, decay):
    import paper_1905_12948_amd as gmc
    n = rows * cols
    w = torch.randn(n, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(5))
    plan = gmc.Matrices(n, [(0, rows, cols)])
    out = gmc.orthogonal_step(plan, w, torch.zeros_like(w), None, 0.02, decay=decay, w_out=torch.empty_like(w)).double()
    want = w.double() * (1 - decay)
    assert ((out - want).abs() <= U * (2 * want.abs() + 2 * abs(decay) * w.double().abs()) + 2.0 ** -149).all()
    if decay in (0.0, 1.0):
        assert torch.equal(out, want)


@pytest.mark.parametrize("decay", [0.0, 0.01, 0.7])
def test_infinite_weights_stay(decay):
    import paper_1905_12948_amd as gmc
    for rows, cols in SHAPES:
        n = rows * cols
        w, u = torch.randn(n, device="cuda:0"), torch.randn(n, device="cuda:0")
        w[5], w[n - 2], w[70] = math.inf, -math.inf, math.nan
        plan = gmc.Matrices(n, [(0, rows, cols)])
        out = gmc.orthogonal_step(plan, w, u, None, 0.02, decay=decay, w_out=torch.empty_like(w))
        assert out[5] == math.inf and out[n - 2] == -math.inf and torch.isnan(out[70])
        assert torch.isfinite(out).sum() == n - 3
