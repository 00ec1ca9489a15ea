"""The 64-bit statements of the worker-side operators against differences of
their own forward formulas, and the dropout mask's rate and independence (CPU)."""
import numpy as np
import pytest

import worker_ref as ref


def slope_of(f, x, at, h=1e-5):
    up, down = x.copy(), x.copy()
    up[at] += h
    down[at] -= h
    return (f(up) - f(down)) / (2 * h)


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("S,C,G", [(5, 6, 2), (1, 8, 1), (7, 4, 4)])
def test_group_norm_gradients_against_differences(kind, S, C, G):
    rng = np.random.default_rng(1)
    x, dy = rng.normal(size=(2, S, C)), rng.normal(size=(2, S, C))
    gamma, beta, eps = 1 + 0.3 * rng.normal(size=C), 0.3 * rng.normal(size=C), 1e-5

    def total(x, gamma, beta):
        return (ref.group_norm(x, G, gamma, beta, eps, kind)[0] * dy).sum()

    _, mean, rstd, _, _ = ref.group_norm(x, G, gamma, beta, eps, kind)
    dx, dgamma, dbeta = ref.group_norm_backward(dy, x, G, gamma, beta, kind, mean, rstd)
    # central differences of a smooth function: error h^2 and rounding / h, both under 1e-6 here;
    # the inputs are fixed and none of their z is within h of relu's corner
    for at in [(0, 0, 0), (1, S - 1, C - 1), (0, S // 2, 1)]:
        assert abs(slope_of(lambda v: total(v, gamma, beta), x, at) - dx[at]) < 1e-6
    for c in range(C):
        assert abs(slope_of(lambda v: total(x, v, beta), gamma, (c,)) - dgamma[c]) < 1e-6
        assert abs(slope_of(lambda v: total(x, gamma, v), beta, (c,)) - dbeta[c]) < 1e-6


@pytest.mark.parametrize("by_sequence", [False, True])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_policy_gradient_against_differences(by_sequence, tau):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(3, 4, 6))
    labels = rng.integers(0, 6, (3, 4))
    labels[0, 0] = labels[2] = ref.IGNORE
    # ratios on both sides of the clip range, for both signs of the advantage
    base = ref.policy(x, labels, None, np.zeros((3, 4)), None, 0.2, 0.2, 0, tau, False)[3]
    old = base - np.array([[0.1, 0.5, -0.5, 0.05]] * 3)
    old_ref = base + 0.3 * rng.normal(size=base.shape)
    adv = np.array([[1.0] * 4, [-1.0] * 4, [1.0] * 4])
    f = lambda v: ref.policy(v, labels, old, adv, old_ref, 0.2, 0.3, 0.1, tau, by_sequence)  # noqa: E731
    grad = f(x)[5]
    for at in [(0, 0, 1), (0, 1, 2), (0, 2, labels[0, 2]), (0, 3, 0), (1, 0, 3), (1, 1, labels[1, 1]), (1, 2, 5), (2, 1, 1)]:
        assert abs(slope_of(lambda v: f(v)[0], x, at) - grad[at]) < 1e-7


@pytest.mark.parametrize("average", [False, True])
def test_preference_gradient_against_differences(average):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(4, 5, 7))
    labels = rng.integers(0, 7, (4, 5))
    labels[0, 3:] = labels[3] = ref.IGNORE
    base = rng.normal(size=(4, 5)) - 2
    f = lambda v: ref.preference(v, labels, base, 0.7, 0.1, average)  # noqa: E731
    grad = f(x)[5]
    for at in [(0, 0, 1), (0, 1, labels[0, 1]), (0, 4, 2), (1, 2, 3), (2, 0, labels[2, 0]), (3, 0, 0)]:
        assert abs(slope_of(lambda v: f(v)[0], x, at) - grad[at]) < 1e-7


def test_dropout_mask_rate_and_independence():
    n = 40_000
    for p in (0.1, 0.5):
        a = ref.dropout_bits(range(n), 7, 3, 0, 0) >= round(65536 * p)
        b = ref.dropout_bits(range(n), 7, 3, 1, 0) >= round(65536 * p)
        c = ref.dropout_bits(range(n), 7, 4, 0, 0) >= round(65536 * p)
        d = ref.dropout_bits(range(n), 7, 3, 0, 1) >= round(65536 * p)
        sd = np.sqrt(p * (1 - p) / n)
        for m in (a, b, c, d):
            assert abs(m.mean() - (1 - p)) < 5 * sd
        for m in (b, c, d):  # other workers, steps and sites: independent masks
            both, sd2 = (1 - p) ** 2, np.sqrt((1 - p) ** 2 * (1 - (1 - p) ** 2) / n)
            assert abs((a & m).mean() - both) < 5 * sd2
        # neighbours share a draw: their bits are independent too
        q = a.reshape(-1, 4)
        assert abs((q[:, 0] & q[:, 1]).mean() - (1 - p) ** 2) < 5 * np.sqrt(0.25 / (n / 4))


def test_the_draws_follow_the_published_stream():
    """State 0's draws are SplitMix64's published first outputs."""
    import os
    path = os.path.join(os.path.dirname(__file__), "golden", "splitmix64_seed0.txt")
    want = [int(v, 0) for line in open(path) for v in line.split("#")[0].split()]
    state0 = ref.mix(1) ^ ref.mix((1 << 32) | 1)  # the seed that makes the stream's state 0
    for j, w in enumerate(want):
        bits = ref.dropout_bits(range(4 * j, 4 * j + 4), state0, 0, 0, 0)
        assert sum(int(b) << (16 * i) for i, b in enumerate(bits)) == w
