"""The worker-side operators' sizes and arguments at the ends of their ranges (no GPU:
nothing here reaches a launch)."""
import ctypes
import os
import time

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


@pytest.mark.parametrize("dtype,N,S,C,G", [(BF16, 2 ** 24, 1, 12, 4), (BF16, 2 ** 26 + 1, 1, 64, 8), (F32, 2 ** 25, 1, 4, 1),
                                           (BF16, 2000, 1, 46523, 46523), (F16, 2 ** 33, 1, 8, 8)])
def test_group_norm_of_more_images_than_a_launch_has_is_taken(lib, dtype, N, S, C, G):
    assert lib.gmc_group_norm_workspace(dtype, N, S, C, G, 0) >= 0
    assert lib.gmc_group_norm_workspace(dtype, N, S, C, G, 1) >= 8 * N * C


P = ctypes.c_void_p(1 << 20)


def refused(lib, st, needle):
    assert st == -1 and needle in lib.gmc_last_error(None).decode(), (st, lib.gmc_last_error(None))


def test_group_norm_of_an_image_no_launch_has_is_refused(lib):
    """By the workspace functions too, and before any other buffer is looked at."""
    C = 2 ** 30
    for backward in (0, 1):
        assert lib.gmc_group_norm_workspace(BF16, 1, 30, C - 1, C - 1, backward) == -1
    refused(lib, lib.gmc_group_norm(None, BF16, 1, 30, C - 1, C - 1, P, 30 * C, C, None, None, 1e-5, 0, P, 30 * C, C, P, P, P,
                                    1 << 50), "launch")
    assert lib.gmc_group_norm_workspace(BF16, 1, 1, C, 1, 1) == -1
    for N in (0, 1):
        Q, R = ctypes.c_void_p(1 << 40), ctypes.c_void_p(1 << 50)
        refused(lib, lib.gmc_group_norm_backward(None, BF16, N, 1, C, 1, R, C, C, P, C, C, P, P, None, None, 0, Q, C, C, P, P, P,
                                                 1 << 50), "launch")


def test_dropout_of_more_vectors_than_a_launch_has_is_refused(lib):
    Q = ctypes.c_void_p(1 << 50)
    refused(lib, lib.gmc_dropout(None, BF16, 2 ** 34 - 1023, 1, P, 2, None, 0, Q, 2, 0.1, 1, 0, 0, 0), "one launch")


def test_a_large_prime_number_of_groups_is_planned_without_a_search_through_them(lib):
    # 2^31 - 1 groups of one channel: 46 s where every number of groups was tried
    at = time.perf_counter()
    lib.gmc_group_norm_workspace(BF16, 1, 1, LAST, LAST, 0)
    assert time.perf_counter() - at < 5


@pytest.mark.parametrize("change,needle", [(dict(kl=1e39), "finite"), (dict(kl=-4e38), "finite"), (dict(scale=1e300), "finite"),
                                           (dict(tau=1e-39), "temperature"), (dict(tau=5e-324), "temperature")])
def test_factors_that_are_infinite_in_32_bits_are_refused(lib, change, needle):
    Q, R = ctypes.c_void_p(1 << 40), ctypes.c_void_p(1 << 50)
    a = dict(dict(kl=0.1, scale=1.0, tau=1.0), **change)
    st = lib.gmc_policy_loss(None, BF16, 4, 3, 10, P, 30, 10, P, 3, -100, None, None, P, 1, 0, 0.2, 0.2, a["kl"], a["tau"], 0,
                             a["scale"], Q, Q, R, 30, 10, None, 0)
    refused(lib, st, needle)
    if "tau" not in change:  # kl is beta here
        st = lib.gmc_preference_loss(None, BF16, 2, 3, 10, P, 30, 10, P, 3, -100, None, a["kl"], 0.0, 0, a["scale"], Q, Q, Q, Q,
                                     R, 30, 10, None, 0)
        refused(lib, st, needle)


def test_loss_workspaces_without_tokens(lib):
    """Sequences without tokens need no more than the sums; pairs beyond what the call takes are refused."""
    least = lib.gmc_policy_loss_workspace(0, 0)
    for R in (1, 2 ** 31, 2 ** 61, 2 ** 63 - 1):
        assert lib.gmc_policy_loss_workspace(R, 0) == least
    assert lib.gmc_preference_loss_workspace(2 ** 21 - 1, 0) == 4 * 2 ** 22
    for pairs in (2 ** 21, 2 ** 31, 2 ** 61, 2 ** 63 - 1):
        assert lib.gmc_preference_loss_workspace(pairs, 0) == -1
        refused(lib, lib.gmc_preference_loss(None, BF16, pairs, 0, 10, None, 30, 10, None, 3, -100, None, 0.1, 0.0, 0, 1.0, P, P,
                                             P, P, None, 30, 10, None, 0), "P < 2^21")
