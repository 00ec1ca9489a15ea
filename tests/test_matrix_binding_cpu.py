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
