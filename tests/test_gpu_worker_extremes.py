"""The losses where a factor of a term is beyond 32 bits or infinite and the other is
zero, and where differences of log-probabilities are small."""
import math

import numpy as np
import pytest

import worker_ref as ref
from test_gpu_worker_ops import LP, U, check, dev, host, logits_gradient_slack

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("V", [9, 5000, 50257, 170001])
def test_ratio_beyond_32_bits_without_advantage(V):
    import paper_1905_12948_amd as gmc
    rng = np.random.default_rng(V)
    R, T = 3, 4
    x, labels = dev(rng.normal(size=(R, T, V))), rng.integers(0, V, (R, T))
    old = dev(np.full((R, T), -1.0) - 200 * (rng.random((R, T)) < 0.5))
    old[1] -= 200
    adv = dev([1.0, 0.0, 0.5])                   # the second sequence: every ratio overflows, A = 0
    A = host(adv)[:, None].repeat(T, 1)
    loss, _, clips, logp, c, grad = ref.policy(host(x), labels, host(old), A, None, 0.2, 0.2, 0, 1.0, False)
    stats, lp, g = gmc.policy_loss(x, torch.as_tensor(labels).cuda(), old, adv)
    elp = LP + 8 * U * np.abs(logp)
    check(lp, logp, elp, "f32", "logp")
    # clipped terms are constants; the others' ratios are e^-(several), off by 16 u and the log-probability's error
    free = np.exp(np.minimum(logp - host(old), 0.2)) * np.abs(A)
    check(stats, np.array([loss, 0, clips]), np.array([((elp + 16 * U) * free).mean() + 8 * U * abs(loss), 0, 8 * U]), "f32", "stats")
    ec = (elp + 16 * U) * 2 * free / (R * T)
    check(g, grad, logits_gradient_slack(c, ec, grad, labels, V), "f32", "gradient")
    assert not g[1].any()


@pytest.mark.parametrize("V", [9, 5000, 50257, 170001])
def test_kl_beyond_32_bits_without_a_coefficient(V):
    import paper_1905_12948_amd as gmc
    torch.manual_seed(V)
    x = torch.randn(3, 4, V, device="cuda:0")
    labels = torch.randint(0, V, (3, 4), device="cuda:0")
    adv = torch.tensor([1.0, -0.5, 0.25], device="cuda:0")
    stats, logp, grad = gmc.policy_loss(x, labels, None, adv)
    refs = logp.clone()
    refs[1, 2] += 300
    refs[2, 0] = math.inf
    watched = gmc.policy_loss(x, labels, None, adv, ref_logp=refs, kl_coef=0.0)
    assert torch.equal(watched[0][[0, 2]], stats[[0, 2]]) and torch.equal(watched[1], logp) and torch.equal(watched[2], grad)


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("P,T", [(2, 3), (9, 60)])
def test_impossible_answers(P, T, average):
    """A rejected answer with a token of probability 0 has lost: without smoothing its
    pair adds 0 and has no gradient.  A chosen one has lost with smoothing 1."""
    import paper_1905_12948_amd as gmc
    V = 30
    torch.manual_seed(P)
    x = torch.randn(2 * P, T, V, device="cuda:0")
    labels = torch.randint(0, V, (2 * P, T), device="cuda:0")
    want = gmc.preference_loss(x, labels, average=average)
    y = x.clone()
    y[P, 1, labels[P, 1]] = -math.inf
    loss, each, rewards, logp, grad = gmc.preference_loss(y, labels, average=average)
    assert rewards[P] == -math.inf and logp[P, 1] == -math.inf
    assert each[0] == 0 and not grad[0].any() and not grad[P].any()
    assert torch.equal(each[1:], want[1][1:]) and torch.equal(grad[1:P], want[4][1:P]) and torch.equal(grad[P + 1:], want[4][P + 1:])
    mean = each.double().sum() / P
    assert abs(loss.double() - mean) <= 4 * U * mean
    assert gmc.preference_loss(y, labels, average=average, smoothing=0.25)[0] == math.inf
    y = x.clone()
    y[0, 1, labels[0, 1]] = -math.inf
    assert gmc.preference_loss(y, labels, average=average)[1][0] == math.inf
    _, each, _, _, grad = gmc.preference_loss(y, labels, average=average, smoothing=1.0)
    assert each[0] == 0 and not grad[0].any() and not grad[P].any() and torch.isfinite(grad).all()


@pytest.mark.parametrize("V", [2, 4096, 65536, 2 ** 18])
@pytest.mark.parametrize("size", [1e-2, 1e-4, 1e-6])
def test_kl_gradient_of_a_reference_close_by(V, size):
    """Without an advantage the gradient is the KL term's, whose slope 1 - e^d is as
    small as the difference d of the log-probabilities.  Rows of equal logits, a power of
    two of them, have a log-probability of -k log 2 without any rounding, so d is known."""
    import paper_1905_12948_amd as gmc
    rng = np.random.default_rng(V)
    R, T, kl = 2, 3, 0.5
    lp = -math.log(V)
    refs = dev(lp + size * rng.choice([-1.0, -0.5, 0.5, 1.0], (R, T)))
    labels = rng.integers(0, V, (R, T))
    _, logp, grad = gmc.policy_loss(torch.zeros(R, T, V, device="cuda:0"), torch.as_tensor(labels).cuda(), None,
                                    torch.zeros(R, device="cuda:0"), ref_logp=refs, kl_coef=kl)
    assert (logp == np.float32(lp)).all()
    c = kl / (R * T) * -np.expm1(host(refs) - lp)
    want = np.repeat(-c[:, :, None] / V, V, 2)
    np.put_along_axis(want, labels[:, :, None], (c * (1 - 1 / V))[:, :, None], 2)
    # relatively: d, its exponential (2 u), three products, the quotient, the product with p, and the label's
    # difference of at least half its larger part: 8 u of at most twice the value
    assert (np.abs(host(grad) - want) <= 16 * U * np.abs(want)).all(), np.abs(host(grad) / want - 1).max() / U
