"""When the binding frees a plan of matrices (no GPU: a library that only notes it)."""
import pytest

torch = pytest.importorskip("torch")
from paper_1905_12948_amd import matrix  # noqa: E402


class Library:
    def __init__(self):
        self.freed = []

    def gmc_matrices_destroy(self, plan):
        self.freed.append(plan)


def test_plans_dropped_during_a_capture_are_freed_after_it(monkeypatch):
    """Freeing waits for the device, which a capture does not allow."""
    library, capturing = Library(), [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])

    def made(number):
        m = object.__new__(matrix.Matrices)
        m._lib, m._plan = library, number
        return m
    one, two, three, four = (made(k) for k in (1, 2, 3, 4))
    one.close()
    assert library.freed == [1] and one._plan is None
    one.close()
    assert library.freed == [1]
    capturing[0] = True
    two.close()
    del three
    assert two._plan is None and library.freed == [1]
    capturing[0] = False
    del four
    assert sorted(library.freed) == [1, 2, 3, 4]
