"""What the binding of the orthogonalised matrices makes of its arguments (no GPU)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_1905_12948_amd import matrix  # noqa: E402


@pytest.mark.parametrize("d,table", [(64.5, []), (64, [(0.5, 4, 4)]), (64, [(0, 4.25, 4)]), (64, [(0, 4, 4, 5.5)]),
                                     (float("nan"), []), (float("inf"), []), (64, [(0, float("inf"), 4)]), ("64", [])])
def test_fractions_are_no_sizes(d, table):
    with pytest.raises(ValueError, match="whole number"):
        matrix.Matrices(d, table)


def test_fractional_steps():
    with pytest.raises(ValueError, match="whole number"):
        matrix._steps(2.5, matrix.QUINTIC)


@pytest.mark.parametrize("v", [7, 7.0, np.int64(7), np.float32(7), torch.tensor(7), torch.tensor(7.0)])
def test_whole_numbers_of_any_type(v):
    got = matrix._whole(v, "d")
    assert got == 7 and type(got) is int


THREE = (3.0, -4.5, 2.0)


@pytest.mark.parametrize("make", [tuple, list, np.array, torch.tensor, lambda v: [torch.tensor(x) for x in v],
                                  lambda v: [np.float32(x) for x in v], lambda v: torch.tensor(v, dtype=torch.float64)])
def test_coefficients_for_all_steps(make):
    n, c = matrix._steps(4, make(THREE))
    assert n == 4 and list(c) == list(THREE) * 4


@pytest.mark.parametrize("make", [list, np.array, torch.tensor, lambda v: [torch.tensor(r) for r in v], lambda v: [np.array(r) for r in v]])
def test_coefficients_of_each_step(make):
    rows = [[3.0, -4.5, 2.0], [1.5, -0.5, 0.0], [1.0, 0.25, 0.5]]
    n, c = matrix._steps(3, make(rows))
    assert n == 3 and list(c) == sum(rows, [])


@pytest.mark.parametrize("bad", [(), (1.0,), (1.0, 2.0), (1.0, 2.0, 3.0, 4.0), [THREE], [THREE] * 3, [(1.0, 2.0)] * 4, 3.0, None,
                                 torch.tensor(1.0), torch.zeros(2), torch.zeros(4, 2), torch.zeros(3, 3), torch.zeros(4, 3, 1)])
def test_other_coefficients(bad):
    with pytest.raises(ValueError, match="coefficients must be"):
        matrix._steps(4, bad)
