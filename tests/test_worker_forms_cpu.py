"""The shapes that group norm is compared at (norm_forms.SHAPES, test_gpu_worker_forms.py)
reach every kernel and every branch of its plan, and the plan stays within its limits."""
import random

import norm_forms as forms
import pytest

LDS = 160 * 1024


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return forms.build(str(tmp_path_factory.mktemp("plan")))


@pytest.mark.parametrize("backward", [0, 1])
def test_every_kernel_is_compared(plan, backward):
    reached = {forms.kernel(plan(size, *shape, backward), size, backward) for size in (2, 4) for shape in forms.SHAPES}
    assert reached == forms.kernels(backward), forms.kernels(backward) - reached


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("size", [2, 4])
def test_every_branch_is_compared(plan, size, backward):
    """Whatever a random call goes through, one of the shapes does too."""
    rng = random.Random(size + backward)
    reached = set()
    for shape in forms.SHAPES:
        reached |= forms.branches(plan(size, *shape, backward), size, *shape, backward)
    for _ in range(30000):
        cpg = rng.choice([1, 1, 2, 4, 8, 16, 32, 64, 3, 5, 12, 17, 96, 131, 256, int(2 ** rng.uniform(0, 11))])
        G = rng.choice([1, 2, 4, 8, 16, 32, 61, 64, 31, int(2 ** rng.uniform(0, 10))])
        shape = int(2 ** rng.uniform(0, 10)), int(2 ** rng.uniform(0, 14)), cpg * G, G
        more = forms.branches(plan(size, *shape, backward), size, *shape, backward) - reached
        assert not more, (more, shape)


def test_plans_are_within_limits(plan):
    """Random calls: every pixel has a place, blocks and pieces make up the image, LDS and
    threads are what a workgroup may have."""
    rng = random.Random(9)
    for _ in range(60000):
        size, backward = rng.choice([2, 4]), rng.randrange(2)
        cpg = rng.choice([1, 2, 4, 8, 16, 32, 64, 3, 5, 12, 17, 96, 131, 256, int(2 ** rng.uniform(0, 16))])
        G = rng.choice([1, 2, 8, 32, 61, 64, int(2 ** rng.uniform(0, 13))])
        C, S, N = cpg * G, int(2 ** rng.uniform(0, 31)), int(2 ** rng.uniform(0, 20))
        p = plan(size, N, S, C, G, backward)
        shape = (size, N, S, C, G, backward, p)
        assert 0 < p["lds"] <= LDS and p["threads"] in (64, 128, 256, 512, 1024) and p["tc"] <= 1 << p["tp_log2"], shape
        rows = p["threads"] >> p["tp_log2"]
        assert rows >= 1
        if p["held"]:
            held = forms.kernel(p, size, backward)[2]
            assert held * rows >= S and p["gw"] * cpg == p["cb"] and p["blocks"] * p["cb"] == C, shape
            assert p["tc"] * p["vec"] == p["cb"] and (not p["fold"] or p["tc"] <= 64), shape
        else:
            assert p["chunks"] * p["chunk"] >= S > (p["chunks"] - 1) * p["chunk"] and p["chunks"] * C < 2 ** 31, shape
            assert p["cblocks"] * p["tc"] * p["vec"] >= C > (p["cblocks"] - 1) * p["tc"] * p["vec"], shape


@pytest.mark.parametrize("size,shape,form", [
    (2, (64, 3136, 256, 32), "split"), (2, (32, 3136, 512, 32), "split"), (4, (64, 3136, 128, 32), "split"),
    (2, (120, 8192, 32, 4), "split"), (2, (16, 3136, 256, 32), "fold"), (2, (1024, 3136, 16, 4), "fold"), (2, (200, 8192, 16, 2), "fold"),
    (2, (4096, 1024, 8, 8), "fold"), (2, (2 ** 19, 8, 8, 2), "fold"), (4, (2048, 4096, 4, 4), "fold"), (4, (2 ** 22, 1, 4, 1), "fold")])
def test_only_blocks_that_share_lines_with_many_give_way_to_a_second_read(plan, size, shape, form):
    """Large images, backward: a block as wide as the image reads whole lines, however narrow."""
    assert forms.kernel(plan(size, *shape, 1), size, 1)[0] == form
