"""Which layouts of matrices gmc_matrices_init takes: all without a shared component, however their rows lie
among each other's, and no other (no GPU: a layout that is taken ends at the missing device)."""
import random

import pytest

from test_scores_refusals_cpu import lib, plan, refused  # noqa: F401 (lib is a fixture)


def shares(table):
    seen = set()
    for offset, rows, cols, pitch in table:
        for r in range(rows):
            for c in range(cols):
                at = offset + r * pitch + c
                if at in seen:
                    return True
                seen.add(at)
    return False


def taken(lib, d, table):  # noqa: F811
    return plan(lib, d, table) == 0 or "share" not in lib.gmc_last_error(None).decode()


@pytest.mark.parametrize("table", [
    [(0, 4, 5, 20), (6, 2, 10, 40)],                    # in every second gap of another
    [(0, 3, 2, 30), (4, 2, 3, 7), (40, 1, 15)],         # whole in the first gap; one row in the second
    [(0, 2, 3, 50), (10, 3, 4, 11)],
    [(5, 1, 3, 9), (0, 2, 4, 9)],                       # a row that runs past another's first one
    [(0, 3, 4, 10), (4, 3, 6, 10)],                     # columns that fill a wide array
])
def test_nested_layouts_are_taken(lib, table):  # noqa: F811
    table = [e if len(e) == 4 else e + (e[2],) for e in table]
    assert not shares(table)
    for order in (table, table[::-1]):
        assert taken(lib, 200, order)


def test_against_every_component(lib):  # noqa: F811
    rng = random.Random(1)
    counts = [0, 0]
    for _ in range(1500):
        table = []
        for _ in range(rng.randint(2, 3)):
            cols, rows = rng.randint(1, 6), rng.randint(1, 4)
            pitch = cols + rng.choice([0, 1, 3, 6, 9, 13])
            table.append((rng.randint(0, 30), rows, cols, pitch))
        both = shares(table)
        counts[both] += 1
        if both:
            refused(lib, plan(lib, 200, table), "share")
        else:
            assert taken(lib, 200, table), table
    assert min(counts) > 200, counts
