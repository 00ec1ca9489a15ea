"""The kernels that batches of pairs with a long vocabulary and large dropouts run on,
against 64-bit statements on the GPU."""
import math

import numpy as np
import pytest

import worker_ref as ref
from test_gpu_worker_ops import HALF, LP, TYPES, U

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def within(got, want, slack, dtype, what):
    """As in test_gpu_worker_ops: the 32-bit error, and half a step of the output's type."""
    rel, least = HALF[dtype]
    got = got.double()
    tol = slack + rel * (want.abs() + slack) + least
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g of the tolerance" % (
        what, bad.sum().item(), bad.numel(), ((got - want).abs() / tol)[bad].max().item())


def pairs(P, T, V, dtype, extra):
    g = torch.Generator(device="cuda:0").manual_seed(V + P + T)
    full = (2 * torch.randn(2 * P, T + extra, V, device="cuda:0", generator=g)).to(TYPES[dtype])
    labels = torch.randint(0, V, (2 * P, T), device="cuda:0", generator=g)
    labels[torch.rand(2 * P, T, device="cuda:0", generator=g) < 0.3] = ref.IGNORE
    labels[1] = ref.IGNORE                       # an empty chosen answer
    labels[P + 2:P + 3, T // 2:] = ref.IGNORE
    refs = -math.log(V) + torch.randn(2 * P, T, device="cuda:0", generator=g)
    return full[:, :T], labels, refs


# more than 8 pairs, or more than 512 tokens on a side, and rows of more than 512 vectors:
# 512 threads a row up to 2048 vectors, 1024 beyond
BATCHES = [("bf16", 9, 3, 5000), ("f16", 9, 3, 16384), ("bf16", 9, 5, 16392), ("bf16", 3, 171, 50257), ("f32", 9, 3, 2500),
           ("f32", 9, 2, 8193), ("f32", 1, 520, 8192), ("f16", 12, 4, 50257), ("f32", 10, 3, 50257), ("bf16", 9, 3, 140001),
           ("bf16", 2, 300, 4104)]


@pytest.mark.parametrize("average,smoothing", [(False, 0.0), (True, 0.1)])
@pytest.mark.parametrize("dtype,P,T,V", BATCHES)
def test_preference_batches(dtype, P, T, V, average, smoothing):
    import paper_1905_12948_amd as gmc
    extra = int(average)                         # a view without each sequence's last token
    x, labels, refs = pairs(P, T, V, dtype, extra)
    beta, scale = 2.0 if average else 0.1, 4096.0 if dtype == "f16" else 1.0
    kept = labels != ref.IGNORE
    y = labels.clamp(min=0)[:, :, None]
    out = gmc.preference_loss(x, labels, refs, beta=beta, smoothing=smoothing, average=average, grad_scale=scale)
    loss, each, rewards, logp, grad = out
    assert grad.shape == x.shape and grad.stride()[1:] == (V, 1)
    # the 64-bit statement, a sequence at a time
    lp = torch.stack([torch.log_softmax(x[r].double(), -1).gather(1, y[r])[:, 0] for r in range(2 * P)]) * kept
    share = 1 / kept.sum(1).clamp(min=1).double() if average else torch.ones(2 * P, device="cuda:0", dtype=torch.float64)
    reward = beta * ((lp - refs.double()) * kept).sum(1) * share
    h = reward[:P] - reward[P:]
    pair = (1 - smoothing) * torch.nn.functional.softplus(-h) + smoothing * torch.nn.functional.softplus(h)
    dh = smoothing * torch.sigmoid(h) - (1 - smoothing) * torch.sigmoid(-h)
    c = torch.cat([dh, -dh]) * beta * share / P
    elp = (LP + 8 * U * lp.abs()) * kept
    er = beta * elp.sum(1) * share + U * reward.abs()
    eh = er[:P] + er[P:]
    within(logp, lp, elp, "f32", "logp")
    within(rewards, reward, er, "f32", "rewards")
    within(each, pair, eh + 4 * U * pair, "f32", "pair losses")
    within(loss, pair.mean(), eh.mean() + 8 * U * pair.mean(), "f32", "loss")
    ec = torch.cat([eh, eh]) * beta * share / (4 * P) + 8 * U * c.abs()
    for r in range(2 * P):
        p = torch.softmax(x[r].double(), -1)
        at = torch.zeros_like(p).scatter_(1, y[r], 1.0)
        want = scale * c[r] * (at - p) * kept[r][:, None]
        size = torch.where(at > 0, torch.ones_like(p), p) * kept[r][:, None]
        within(grad[r], want, scale * (ec[r] + 2 * LP * c[r].abs()) * size, dtype, "gradient of sequence %d" % r)
    assert not grad[~kept].any()
    # over the logits, whatever lies in the gaps of a view; the same bits again
    full = torch.empty_strided((2 * P, T + extra, V), ((T + extra) * V, V, 1), dtype=x.dtype, device=x.device).fill_(3.0)
    z = full[:, :T]
    z.copy_(x)
    over = gmc.preference_loss(z, labels, refs, beta=beta, smoothing=smoothing, average=average, grad_scale=scale, out=z)
    for a, b in zip(over, out):
        assert torch.equal(a, b)
    assert (full[:, T:] == 3.0).all()
    # the ignored tokens' logits are not looked at
    z.copy_(x)
    z[~kept] = math.nan
    for a, b in zip(gmc.preference_loss(z, labels, refs, beta=beta, smoothing=smoothing, average=average, grad_scale=scale), out):
        assert torch.equal(a, b)


def bits(n, seed, t, worker, site):
    """The mask's 16 bits of elements 0 .. n - 1, on the GPU in wrapping 64-bit integers."""
    def signed(z):
        z &= ref.M64
        return z - (1 << 64) if z >> 63 else z

    def mix(z):
        z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * signed(0xBF58476D1CE4E5B9)
        z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * signed(0x94D049BB133111EB)
        return z ^ ((z >> 31) & ((1 << 33) - 1))
    state = seed ^ ref.mix(t + 1) ^ ref.mix(((worker + 1) << 32) | (site + 1))
    draw = mix(torch.arange(1, n // 4 + 2, device="cuda:0") * signed(0x9E3779B97F4A7C15) + signed(state))
    return ((draw[:, None] >> torch.arange(0, 64, 16, device="cuda:0")) & 65535).reshape(-1)[:n]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,pitch", [(9001, 2048, 2048), (17000, 1001, 1001), (17000, 1001, 1024), (20003, 1030, 1033),
                                             (2200000, 7, 9), (700001, 31, 32)])
def test_large_dropouts(rows, cols, pitch, dtype):
    """Calls of more than 2^21 vectors, by four a thread: with a residual and without, pitched,
    in odd columns, in place."""
    import paper_1905_12948_amd as gmc
    assert rows * -(-cols * (4 if dtype == "f32" else 2) // 16) >= 2 ** 21
    g = torch.Generator(device="cuda:0").manual_seed(cols)
    x = torch.randn(rows, pitch, device="cuda:0", generator=g).to(TYPES[dtype])[:, :cols]
    r = torch.randn(rows, pitch, device="cuda:0", generator=g).to(TYPES[dtype])[:, :cols]
    where = dict(seed=77, t=3, worker=5, site=1)
    p = 0.3
    level = math.floor(65536 * p + 0.5)
    keep = (bits(rows * cols, **where) >= level).view(rows, cols)
    # the same bits as the statement in Python integers
    for i in (0, 5, rows * cols // 2 + 3, rows * cols - 1):
        assert ref.dropout_bits([i], 77, 3, 5, 1)[0] >= level if keep.view(-1)[i] else ref.dropout_bits([i], 77, 3, 5, 1)[0] < level
    value = x.double() * keep * (65536 / (65536 - level))
    plain = gmc.dropout(x, p, **where)
    # scale, product, sum: three roundings of at most |x| scale + |r|
    within(plain, value, 2 * U * value.abs(), dtype, "dropout")
    joined = gmc.dropout(x, p, residual=r, **where)
    within(joined, value + r.double(), 3 * U * (value.abs() + r.double().abs()), dtype, "dropout and residual")
    if pitch > cols:
        wide = torch.zeros(rows, pitch, device="cuda:0", dtype=TYPES[dtype])
        v = wide[:, :cols]
        v.copy_(x)
        gmc.dropout(v, p, residual=r, out=v, **where)
        assert torch.equal(v, joined) and not wide[:, cols:].any()
    else:
        y = r.clone()
        assert torch.equal(gmc.dropout(x, p, residual=y, out=y, **where), joined)


# each class of rows that policy_held has, at its ends: 512, 2048, 4096, 6656, 13312 and 20480 vectors
@pytest.mark.parametrize("dtype,V", [("bf16", 4104), ("bf16", 16384), ("f16", 16392), ("f16", 32768), ("bf16", 32776), ("bf16", 53248),
                                     ("f16", 53256), ("bf16", 106496), ("f16", 106504), ("bf16", 163840), ("f32", 2048), ("f32", 2052),
                                     ("f32", 8192), ("f32", 8196), ("f32", 16384), ("f32", 16388), ("f32", 26624), ("f32", 26628),
                                     ("f32", 53248), ("f32", 53252), ("f32", 81920)])
def test_policy_rows_at_the_ends_of_their_classes(dtype, V):
    from test_gpu_worker_ops import test_policy_loss
    test_policy_loss(V, dtype)
