"""Matrices between other matrices' rows (gmc_orthogonalize, gmc_orthogonal_step): each comes out as it
does alone, and what lies between them stays.

Alone a matrix may go through other launches (one workgroup's, or tiles of another size), whose sums have
another order.  A sum of up to 350 terms is then off by sqrt(350 / 16 * 3) 2^-24 of its terms' norms and kept values by 2^-22, ten
times (five steps' X and polynomial), amplified as small values are: 485 of errors that are each 2^-21 of
an entry's share (1 / 30 of the largest): 485 sqrt(10) 2^-21 / 30 = 2.4e-5 of the largest entry."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# (offset, rows, cols, pitch), within 40,000 components
LAYOUTS = [
    [(7, 30, 40, 400), (60, 15, 300, 800), (450, 14, 350, 800)],      # in every second gap, either kind
    [(0, 3, 50, 9000), (100, 70, 60, 99), (9060, 1, 500), (9600, 60, 90)],    # whole within a gap
    [(11, 200, 33, 190), (44, 200, 100, 190), (144, 200, 57, 190)],   # every column of a wide array
]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
@pytest.mark.parametrize("order", [1, -1])
def test_nested_matrices(layout, order):
    import paper_1905_12948_amd as gmc
    d, table = 40000, [e if len(e) == 4 else e + (e[2],) for e in LAYOUTS[layout]][::order]
    x, w, m = (torch.randn(d, device="cuda:0") for _ in range(3))
    plan = gmc.Matrices(d, table)
    out, past, into = gmc.orthogonalize(plan, x), m.clone(), torch.empty_like(w)
    gmc.orthogonal_step(plan, w, x, past, 0.1, mu=0.9, decay=0.01, w_out=into)
    want, want_past, want_into = x.clone(), m.clone(), w + x
    for offset, rows, cols, pitch in table:
        def view(t):
            return torch.as_strided(t, (rows, cols), (pitch, 1), offset)
        one = gmc.Matrices(rows * cols, [(0, rows, cols)])
        a, b, c = (view(t).contiguous().view(-1) for t in (x, w, m))
        view(want).copy_(gmc.orthogonalize(one, a).view(rows, cols))
        view(want_into).copy_(gmc.orthogonal_step(one, b, a, c, 0.1, mu=0.9, decay=0.01).view(rows, cols))
        view(want_past).copy_(c.view(rows, cols))
    for got, exact in ((out, want), (into, want_into)):
        assert (got - exact).abs().max() < 2.4e-5 * exact.abs().max()
    free = torch.ones(d, dtype=torch.bool, device="cuda:0")
    for offset, rows, cols, pitch in table:
        torch.as_strided(free, (rows, cols), (pitch, 1), offset).fill_(False)
    assert free.any() and torch.equal(out[free], x[free]) and torch.equal(past, want_past)
    assert torch.equal(into[free], (w + x)[free])
