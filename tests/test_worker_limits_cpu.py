"""The worker-side operators' sizes and arguments at the ends of their ranges (no GPU:
nothing here reaches a launch)."""
import os

import pytest

F32, BF16, F16 = 0, 1, 2
LAST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    from paper_1905_12948_amd import gmc
    if not os.path.exists(gmc.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return gmc.load()


@pytest.mark.parametrize("C,G", [(1, 1), (3, 1), (8, 4), (136, 1)])
@pytest.mark.parametrize("backward", [0, 1])
def test_group_norm_workspace_up_to_the_last_number_of_pixels(lib, C, G, backward):
    # images this long are summed in pieces, whose number, and so the scratch, grows with them
    sizes = [LAST - 40000, LAST - 16384, LAST - 16383, LAST - 16382, LAST - 2048, LAST - 255, LAST - 1, LAST]
    need = [lib.gmc_group_norm_workspace(BF16, 1, S, C, G, backward) for S in sizes]
    assert need[0] >= 2 * 4 * C * (sizes[0] // 16384) and need == sorted(need), need


def test_group_norm_workspace_of_wide_long_images(lib):
    # 2^37 values an image: chunks times channels stay below 2^31, two fp32 sums each
    for S, C in [(2 ** 17, 2 ** 20), (2 ** 20, 2 ** 17), (2 ** 25, 2 ** 12)]:
        need = lib.gmc_group_norm_workspace(BF16, 1, S, C, 1, 0)
        assert 0 < need <= 2 * 4 * LAST, (S, C, need)
