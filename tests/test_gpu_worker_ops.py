"""The worker-side operators on the GPU against their 64-bit statements
(worker_ref.py).

Tolerances, with u = 2^-24 (one 32-bit rounding): a 16-bit output is the 32-bit
result rounded once, so it is within half a step of its type (at most 2^-8 of the
value for bfloat16's 8 bits, 2^-11 or half of 2^-24 for float16's 11; the latter
doubled here) plus the 32-bit error.  The 32-bit bounds are
worst cases of the operations each result goes through, named at each check."""
import math

import numpy as np
import pytest

import worker_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -24)}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(a, dtype="f32"):
    return torch.as_tensor(np.asarray(a, np.float32)).to("cuda:0").to(TYPES[dtype])


def host(t):
    return t.detach().double().cpu().numpy()


def check(got, want, slack, dtype, what):
    """|got - want| <= slack (32-bit error) + the output's own rounding."""
    rel, least = HALF[dtype]
    got = host(got)
    tol = slack + rel * (np.abs(want) + slack) + least
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g at tolerance %g" % (
        what, bad.sum(), bad.size, np.abs(got - want)[bad].max(), np.broadcast_to(tol, bad.shape)[bad].min())


# -- dropout ----------------------------------------------------------------


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,pitch", [(1, 1, 1), (1, 7, 7), (3, 5, 5), (5, 9, 12), (2, 64, 64), (7, 33, 40), (4, 1001, 1024),
                                             (300, 10, 11)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(dtype, rows, cols, pitch, p):
    import paper_1905_12948_amd as gmc
    rng = np.random.default_rng(rows * cols)
    x = dev(rng.normal(size=(rows, pitch)), dtype)[:, :cols]
    r = dev(rng.normal(size=(rows, pitch)), dtype)[:, :cols]
    at = dict(seed=2 ** 63 + 5, t=9, worker=3, site=2)
    scale = 65536 / (65536 - math.floor(65536 * p + 0.5)) if p < 1 else 0
    for residual in (None, r):
        want, keep = ref.dropout(host(x), p, 2 ** 63 + 5, 9, 3, 2, None if residual is None else host(r))
        got = gmc.dropout(x, p, residual=residual, **at)
        # scale, product, sum: three roundings of at most |x| scale + |r|
        slack = 3 * U * (np.abs(host(x)) * scale + (0 if residual is None else np.abs(host(r))))
        check(got, want, slack, dtype, "dropout")
        if residual is None:
            assert np.array_equal(host(got) != 0, keep & (host(x) != 0))
    back = gmc.dropout_backward(r, p, **at)
    want, _ = ref.dropout(host(r), p, 2 ** 63 + 5, 9, 3, 2)
    check(back, want, 3 * U * np.abs(want), dtype, "dropout backward")
    if p < 1:  # the mask of the forward call, whatever the layout
        assert torch.equal(gmc.dropout(torch.ones_like(x), p, **at) != 0, gmc.dropout_backward(torch.ones_like(r), p, **at) != 0)


def test_dropout_in_place_and_nan():
    import paper_1905_12948_amd as gmc
    x = torch.randn(37, 50, device="cuda:0", dtype=torch.bfloat16)
    r = torch.randn_like(x)
    want = gmc.dropout(x, 0.3, 5, residual=r)
    a, b = x.clone(), r.clone()
    assert torch.equal(gmc.dropout(a, 0.3, 5, residual=r, out=a), want)
    assert torch.equal(gmc.dropout(x, 0.3, 5, residual=b, out=b), want)
    wide = torch.zeros(37, 64, device="cuda:0", dtype=torch.bfloat16)
    gmc.dropout(x, 0.3, 5, residual=r, out=wide[:, 7:57])
    assert torch.equal(wide[:, 7:57], want) and not wide[:, :7].any() and not wide[:, 57:].any()
    mask = gmc.dropout(torch.ones_like(x), 0.3, 5) == 0
    y = gmc.dropout(x.masked_fill(mask, float("nan")), 0.3, 5, residual=r)
    assert torch.equal(y, want)
    # three axes, and a view whose rows are evenly spaced
    z = torch.randn(3, 4, 20, device="cuda:0")
    assert torch.equal(gmc.dropout(z[:, :, :9], 0.3, 5), gmc.dropout(z[:, :, :9].contiguous(), 0.3, 5))
    with pytest.raises(ValueError):
        gmc.dropout(z[:, :2, :9], 0.3, 5)
    assert gmc.dropout(z[:0], 0.3, 5).shape == (0, 4, 20)


def test_dropout_far_offsets():
    """Elements beyond 2^32 of a call, contiguous and by pitch."""
    import paper_1905_12948_amd as gmc
    n = 2 ** 32 + 4099
    x = torch.ones(n, device="cuda:0", dtype=torch.bfloat16)
    y = gmc.dropout(x, 0.5, 11, t=1)
    for first in (0, 2 ** 31 - 50, 2 ** 32 - 50, n - 100):
        want, _ = ref.dropout(np.ones(100), 0.5, 11, 1, 0, 0, first=first)
        assert np.array_equal(host(y[first:first + 100]), want), first
    del y
    pitch = 2 ** 31 + 3
    v = x.as_strided((2, 301), (pitch, 1))
    want, _ = ref.dropout(np.ones((2, 301)), 0.5, 11, 1, 0, 0)
    assert np.array_equal(host(gmc.dropout(v, 0.5, 11, t=1)), want)


# -- group norm --------------------------------------------------------------

NORMS = [  # N, S, C, G: every form (held with few and many pixels, wide blocks, one channel a thread; split)
    (2, 7, 8, 2), (1, 1, 64, 1), (3, 5, 3, 1), (2, 49, 12, 4), (2, 49, 96, 32), (2, 300, 64, 32), (1, 1024, 64, 8),
    (3, 4, 2048, 1), (2, 33, 2048, 32), (1, 900, 40, 5), (2, 1500, 256, 2), (1, 5000, 9, 1), (2, 2100, 136, 1),
    (1, 700, 4104, 1), (5, 2, 131, 131)]


def norm_case(N, S, C, dtype, level=1.0):
    rng = np.random.default_rng(N * S + C)
    x = dev(rng.normal(size=(N, S, C)) * np.exp(0.5 * rng.normal(size=C)) + level * rng.normal(size=C), dtype)
    gamma, beta = dev(1 + 0.3 * rng.normal(size=C)), dev(0.3 * rng.normal(size=C))
    return x, gamma, beta, dev(rng.normal(size=(N, S, C)), dtype)


def norm_slack(x, mean, rstd, G, S, C):
    """(error of hat, size of hat's parts): the mean of m values summed in runs of at
    most 64 and then by halves is off by at most 100 u of the mean size of its terms, and
    so relatively is the variance; then one rounding each for difference and product."""
    N = x.shape[0]
    v = np.abs(x.reshape(N, S, G, -1))
    size = (v + np.abs(mean)[:, None, :, None]) * rstd[:, None, :, None]
    most = v.mean((1, 3), keepdims=True) * rstd[:, None, :, None]
    hat = np.abs(x.reshape(N, S, G, -1) - mean[:, None, :, None]) * rstd[:, None, :, None]
    err = U * (100 * most + 4 * size + 110 * hat)
    return err.reshape(x.shape)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("N,S,C,G", NORMS)
def test_group_norm_forward(N, S, C, G, kind, dtype):
    import paper_1905_12948_amd as gmc
    x, gamma, beta, _ = norm_case(N, S, C, dtype)
    y, mean, rstd = gmc.group_norm(x, G, gamma, beta, act=kind)
    g, b = host(gamma), host(beta)
    want, m, r, hat, z = ref.group_norm(host(x), G, g, b, 1e-5, kind)
    size = np.abs(host(x)).reshape(N, S, G, -1).mean((1, 3))
    check(mean, m, 100 * U * size, "f32", "mean")
    check(rstd, r, 110 * U * r, "f32", "rstd")
    # the activations' slopes stay below 1.1; silu's own exp, sum, reciprocal and product add 8 u
    # and the exponent's argument 2 u |z|
    slack = 1.1 * (norm_slack(host(x), m, r, G, S, C) * np.abs(g) + 2 * U * (np.abs(hat * g) + np.abs(b)))
    check(y, want, slack + (U * np.abs(z) * (8 + 2 * np.abs(z)) if kind == "silu" else 0), dtype, "y")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("N,S,C,G", NORMS)
def test_group_norm_backward(N, S, C, G, kind, dtype):
    import paper_1905_12948_amd as gmc
    x, gamma, beta, dy = norm_case(N, S, C, dtype)
    g, b = host(gamma), host(beta)
    _, mean, rstd = gmc.group_norm(x, G, gamma, beta, act=kind)
    dx, dgamma, dbeta = gmc.group_norm_backward(dy, x, mean, rstd, gamma, beta, act=kind)
    m, r = host(mean), host(rstd)
    if kind == "relu":  # z within rounding of relu's corner may fall on either side: the kernel's own side is used
        hat32 = (x.float().reshape(N, S, G, -1) - mean[:, None, :, None]) * rstd[:, None, :, None]
        z32 = hat32.reshape(N, S, C) * gamma + beta
        on, kind64 = host(z32 > 0), "none"
    else:
        on, kind64 = 1.0, kind
    want, wg, wb = ref.group_norm_backward(host(dy) * on, host(x), G, g, b, kind64, m, r)
    _, _, _, hat, z = ref.group_norm(host(x), G, g, b, 0.0, kind64, m, r)
    dz = np.abs(host(dy) * on * ref.act_slope(z, kind64))
    # dz is off by 20 u of |dy| (1 + |z|) (silu: its gate, products and sums; u |z| through the
    # exponent and u |hat gamma| through z), hat by 4 u of its parts
    ez = U * (20 * np.abs(host(dy)) * (1 + np.abs(z)) + 4 * np.abs(host(dy))) if kind == "silu" else U * dz
    parts = (np.abs(host(x)) + np.abs(m).repeat(C // G, 1)[:, None, :]) * r.repeat(C // G, 1)[:, None, :]
    ez = ez + (U * 4 * parts * np.abs(g) * np.abs(host(dy)) if kind == "silu" else 0)
    eh = 4 * U * parts
    # sums over images and pixels: runs of at most 2048 / 8 ... 64 terms, then by halves: 200 u of the sum of sizes
    check(dbeta, wb, (ez + 200 * U * dz).sum((0, 1)), "f32", "dbeta")
    check(dgamma, wg, (ez * np.abs(hat) + dz * eh + 200 * U * dz * np.abs(hat)).sum((0, 1)), "f32", "dgamma")
    M = S * (C // G)
    grp = lambda a: a.reshape(N, S, G, -1).sum((1, 3), keepdims=True) / M  # noqa: E731
    w, ah, ag = (dz * np.abs(g)).reshape(N, S, G, -1), np.abs(hat).reshape(N, S, G, -1), np.abs(g)
    s1, s2 = grp(w), grp(w.reshape(N, S, C) * np.abs(hat))
    e1 = grp((ez + 250 * U * dz) * ag)
    e2 = grp((ez * np.abs(hat) + dz * eh + 250 * U * dz * np.abs(hat)) * ag)
    err = (ez * ag).reshape(w.shape) + e1 + ah * e2 + eh.reshape(w.shape) * s2 + 6 * U * (w + s1 + ah * s2)
    check(dx, want, (r[:, None, :, None] * err).reshape(N, S, C), dtype, "dx")


@pytest.mark.parametrize("S,C,G", [(64, 64, 8), (2100, 136, 1)])
def test_group_norm_level_far_above_spread(S, C, G):
    """A mean a thousand times the spread: the variance is taken about the mean."""
    import paper_1905_12948_amd as gmc
    rng = np.random.default_rng(S)
    x = dev(1000 + rng.normal(size=(2, S, C)))
    y, mean, rstd = gmc.group_norm(x, G)
    want, m, r, _, _ = ref.group_norm(host(x), G, 1.0, 0.0, 1e-5, "none")
    check(mean, m, 100 * U * np.abs(m), "f32", "mean")
    # an error e of the mean adds e^2 to the variance and e times the level's rounding: far below 200 u here
    check(rstd, r, 4 * 200 * U * r, "f32", "rstd")
    check(y, want, 4 * norm_slack(host(x), m, r, G, S, C), "f32", "y")


def test_group_norm_layouts():
    import paper_1905_12948_amd as gmc
    torch.manual_seed(0)
    for S, C, G in [((6, 5), 24, 3), ((50, 45), 136, 1)]:
        # a torch convolution's channels-last result
        nchw = torch.randn(2, C, *S, device="cuda:0").to(memory_format=torch.channels_last)
        x = nchw.permute(0, 2, 3, 1)
        gamma, beta = torch.randn(C, device="cuda:0"), torch.randn(C, device="cuda:0")
        y, mean, rstd = gmc.group_norm(x, G, gamma, beta, act="relu")
        dy = torch.randn_like(y)
        dx, dg, db = gmc.group_norm_backward(dy, x, mean, rstd, gamma, beta, act="relu")
        # channels of a wider buffer, images apart
        wide = torch.randn(4, *S, C + 13, device="cuda:0")
        v = wide[::2, :, :, 5:5 + C]
        v.copy_(x)
        y2, m2, r2 = gmc.group_norm(v, G, gamma, beta, act="relu")
        assert torch.equal(y2, y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
        keep = wide.clone()
        gmc.group_norm(v, G, gamma, beta, act="relu", out=v)
        keep[::2, :, :, 5:5 + C] = y
        assert torch.equal(wide, keep)
        v.copy_(dy)
        row = torch.zeros(2 * C + 6, device="cuda:0")
        dx2, dg2, _ = gmc.group_norm_backward(v, x, mean, rstd, gamma, beta, act="relu", out=v, dgamma=row[3:3 + C],
                                              dbeta=row[3 + C:3 + 2 * C])
        assert torch.equal(dx2, dx) and torch.equal(dg2, dg) and torch.equal(row[3 + C:3 + 2 * C], db)
        assert not row[:3].any() and not row[-3:].any()
    with pytest.raises(ValueError):
        gmc.group_norm(nchw, G)
    with pytest.raises(ValueError):
        gmc.group_norm(x[:, ::2, ::2], G)
    with pytest.raises(gmc.GmcError):
        gmc.group_norm(x, 7)
    none = x[:0]
    y, mean, rstd = gmc.group_norm(none, G, gamma, beta)
    _, dg, db = gmc.group_norm_backward(none, none, mean, rstd, gamma, beta)
    assert not dg.any() and not db.any()


def test_group_norm_far_offsets():
    """Images more than 2^32 bytes apart."""
    import paper_1905_12948_amd as gmc
    for S, C, G in [(9, 64, 8), (2100, 136, 1)]:
        buf = torch.empty(2 ** 31 + S * C, device="cuda:0", dtype=torch.bfloat16)
        v = buf.as_strided((2, S, C), (2 ** 31, C, 1))
        x = torch.randn(2, S, C, device="cuda:0").bfloat16()
        v.copy_(x)
        want = gmc.group_norm(x, G)
        for a, b in zip(gmc.group_norm(v, G), want):
            assert torch.equal(a, b)
        for a, b in zip(gmc.group_norm_backward(x, v, *want[1:]), gmc.group_norm_backward(x, x, *want[1:])):
            assert torch.equal(a, b)


# -- losses --------------------------------------------------------------------

LP = 250 * U    # relative error of a softmax value: sums of runs of up to 128, the waves, exp, the argument's 3 u |d|
VOCABS = [1, 2, 17, 255, 4097, 16500, 50257, 65600]


def loss_case(R, T, V, dtype, seed, extra=0, pad=0):
    rng = np.random.default_rng(seed)
    data = np.full((R, T + extra, V + pad), 50.0, np.float32)
    data[:, :, :V] = 2 * rng.normal(size=(R, T + extra, V))
    x = dev(data, dtype)[:, :T, :V]
    labels = rng.integers(0, V, (R, T))
    labels[0, :T // 2] = ref.IGNORE
    labels[-1] = ref.IGNORE
    return rng, x, labels


def logits_gradient_slack(c, ec, want_grad, labels, V):
    """c (delta - p): c's error at the label, and p's relative error with c's at each entry."""
    delta = np.zeros(want_grad.shape)
    r, t = np.nonzero(labels != ref.IGNORE)
    delta[r, t, labels[r, t]] = 1
    c, ec = np.abs(c)[:, :, None], ec[:, :, None]
    p = np.abs(np.divide(want_grad, c, out=np.zeros_like(want_grad), where=c > 0))
    p = np.where(delta > 0, 1.0, p)
    return (ec + (2 * LP) * c) * p


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", VOCABS)
def test_policy_loss(V, dtype):
    import paper_1905_12948_amd as gmc
    R, T = (4, 5) if V < 1000 else (3, 3)
    by_seq, tau, kl = V % 2 == 0, 0.8 if V in (17, 50257) else 1.0, 0.1 if V != 255 else 0.0
    rng, x, labels = loss_case(R, T, V, dtype, V, extra=1, pad=3)
    base = ref.policy(host(x), labels, None, np.zeros((R, T)), None, 0, 0, 0, tau, False)[3]
    # ratios inside and outside the clip range, none within rounding of its ends
    old = dev(base - rng.choice([-0.5, -0.1, 0.02, 0.4], (R, T)))
    refs = dev(base + 0.3 * rng.normal(size=(R, T))) if kl else None
    per_token = V % 3 == 0
    adv = dev(rng.normal(size=(R, T) if per_token else R))
    A = host(adv) if per_token else host(adv)[:, None].repeat(T, 1)
    scale = 4096.0 if dtype == "f16" else 1.0
    loss, kls, clips, logp, c, grad = ref.policy(host(x), labels, host(old), A, None if refs is None else host(refs),
                                                 0.2, 0.3, kl, tau, by_seq)
    got = gmc.policy_loss(x, torch.as_tensor(labels).cuda(), old, adv, ref_logp=refs, clip=(0.2, 0.3), kl_coef=kl,
                          temperature=tau, reduction="sequence" if by_seq else "token", grad_scale=scale)
    kept = labels != ref.IGNORE
    elp = np.where(kept, LP + 8 * U * np.abs(logp), 0.0)
    check(got[1], logp, elp, "f32", "logp")
    d = 0 if refs is None else np.abs(np.expm1(host(refs) - logp))
    ratio = np.exp(logp - host(old))
    weight = np.where(kept, 1.0, 0.0) / (kept.sum() if not by_seq else np.maximum(kept.sum(1, keepdims=True), 1) * (kept.sum(1) > 0).sum())
    # the loss's slope in logp is at most ratio |A| + kl |e^d - 1|, and each term is a few roundings
    eloss = (weight * (elp + 16 * U) * (ratio * np.abs(A) + kl * (d + 1))).sum() + 8 * U * abs(loss)
    ekl = (weight * (elp + 16 * U) * (d + 1)).sum()
    check(got[0], np.array([loss, kls, clips]), np.array([eloss, ekl, 8 * U]), "f32", "stats")
    ec = weight * (elp + 16 * U) * (2 * ratio * np.abs(A) + kl * (2 * d + 1))
    check(got[2], scale * grad, scale / tau * logits_gradient_slack(c, ec, grad * tau, labels, V), dtype, "gradient")
    assert not host(got[2])[~kept].any()
    # without the gradient, and the same bits again
    alone = gmc.policy_loss(x, torch.as_tensor(labels).cuda(), old, adv, ref_logp=refs, clip=(0.2, 0.3), kl_coef=kl,
                            temperature=tau, reduction="sequence" if by_seq else "token", grad=False)
    assert alone[2] is None and torch.equal(alone[0], got[0]) and torch.equal(alone[1], got[1])


@pytest.mark.parametrize("dtype,V", [("f32", 65537 + 8), ("bf16", 131072 + 20), ("f16", 140001)])
def test_policy_loss_long_vocabulary(dtype, V):
    test_policy_loss.__wrapped__(V, dtype) if hasattr(test_policy_loss, "__wrapped__") else test_policy_loss(V, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", VOCABS + [140001])
def test_preference_loss(V, dtype):
    import paper_1905_12948_amd as gmc
    P, T = (3, 5) if V < 1000 else (2, 2)
    average, smoothing, beta = V % 2 == 0, 0.1 if V % 3 else 0.0, 0.5
    rng, x, labels = loss_case(2 * P, T, V, dtype, V + 1, extra=1, pad=5)
    base = ref.preference(host(x), labels, None, beta, smoothing, average)[3]
    refs = dev(np.where(labels == ref.IGNORE, np.nan, base + 0.5 * rng.normal(size=base.shape)))
    scale = 1024.0 if dtype == "f16" else 1.0
    with np.errstate(invalid="ignore"):
        loss, each, rewards, logp, c, grad = ref.preference(host(x), labels, host(refs), beta, smoothing, average)
    got = gmc.preference_loss(x, torch.as_tensor(labels).cuda(), refs, beta=beta, smoothing=smoothing, average=average,
                              grad_scale=scale)
    kept = labels != ref.IGNORE
    elp = np.where(kept, LP + 8 * U * np.abs(logp), 0.0)
    share = 1 / np.maximum(kept.sum(1), 1) if average else np.ones(2 * P)
    er = beta * elp.sum(1) * share + U * np.abs(rewards)
    eh = er[:P] + er[P:]
    check(got[3], logp, elp, "f32", "logp")
    check(got[2], rewards, er, "f32", "rewards")
    check(got[1], each, eh + 4 * U * np.abs(each), "f32", "pair losses")  # the loss's slope in h is below 1
    check(got[0], loss, eh.mean() + 8 * U * abs(loss), "f32", "loss")
    # c's slope in h is at most beta share / (4 P)
    ec = np.concatenate([eh, eh]) * beta * share / (4 * P) + 8 * U * np.abs(c)
    rows = np.ones((1, T))
    check(got[4], scale * grad, scale * logits_gradient_slack(c[:, None] * rows, ec[:, None] * rows, grad, labels, V), dtype, "gradient")
    assert not host(got[4])[~kept].any()
    alone = gmc.preference_loss(x, torch.as_tensor(labels).cuda(), refs, beta=beta, smoothing=smoothing, average=average, grad=False)
    assert alone[4] is None and all(torch.equal(a, b) for a, b in zip(alone[:4], got[:4]))


def both_losses(x, labels, out=None, **more):
    """Both losses' results on one set of logits, as a flat list."""
    import paper_1905_12948_amd as gmc
    R = x.shape[0]
    adv = torch.linspace(-1, 1, R, device=x.device)
    a = gmc.policy_loss(x.clone() if out else x, labels, None, adv, **more) if not out else None
    if out:
        y = x.clone()
        a = gmc.policy_loss(y, labels, None, adv, out=y, **more)
        assert a[2] is y
        y = x.clone()
        b = gmc.preference_loss(y, labels, out=y)
        assert b[4] is y
    else:
        b = gmc.preference_loss(x, labels)
    return [*a, *b]


@pytest.mark.parametrize("V", [33, 5000, 50257, 140001])
def test_losses_over_the_logits(V):
    torch.manual_seed(V)
    x = torch.randn(4, 3, V, device="cuda:0").bfloat16()
    labels = torch.randint(0, V, (4, 3), device="cuda:0")
    labels[1, 0] = labels[2] = ref.IGNORE
    for a, b in zip(both_losses(x, labels), both_losses(x, labels, out=True)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("V", [33, 5000, 50257, 140001])
def test_losses_masked_and_odd_values(V):
    """-inf and the type's lowest value among the logits, ignored tokens holding NaN, rows
    all at the lowest value, a row with a NaN, a label out of range."""
    import paper_1905_12948_amd as gmc
    torch.manual_seed(V)
    for dtype in TYPES.values():
        x = torch.randn(2, 6, V, device="cuda:0").to(dtype)
        labels = torch.randint(0, V - 9, (2, 6), device="cuda:0")
        x[:, :, V - 9:] = -math.inf
        x[:, 1, V - 9:] = torch.finfo(dtype).min
        x[0, 2] = torch.finfo(dtype).min
        x[0, 3] = math.nan
        labels[0, 3] = ref.IGNORE
        want = ref.policy(host(x), labels.cpu().numpy(), None, np.ones((2, 6)), None, 0.2, 0.2, 0, 1.0, False)
        stats, logp, grad = gmc.policy_loss(x, labels, None, torch.ones(2, device="cuda:0"))
        lp = host(logp)
        assert np.all(np.abs(lp - want[3]) <= LP + 8 * U * np.abs(want[3]))
        assert abs(lp[0, 2] + math.log(V)) < 1e-5      # uniform over the whole row
        assert not host(grad)[0, 3].any() and not host(grad)[:, 0, V - 9:].any() and not host(grad)[:, 1, V - 9:].any()
        assert torch.isfinite(grad).all() and torch.isfinite(stats).all()
        pref = gmc.preference_loss(x, labels)
        assert torch.isfinite(pref[4]).all()
        assert np.all(np.abs(host(pref[3]) - want[3]) <= LP + 8 * U * np.abs(want[3]))
        # one bad token shows in its own row and in the loss, and nowhere else
        for spoil in ("nan", "inf", "label", "all -inf"):
            y, l2 = x.clone(), labels.clone()
            if spoil == "label":
                l2[1, 4] = V
            elif spoil == "all -inf":
                y[1, 4] = -math.inf
            else:
                y[1, 4, V // 2] = float(spoil)
            s2, p2, g2 = gmc.policy_loss(y, l2, None, torch.ones(2, device="cuda:0"))
            assert torch.isnan(s2[0]) and torch.isnan(p2[1, 4]) and torch.isnan(g2[1, 4]).all(), spoil
            g2[1, 4] = 0
            assert torch.isfinite(g2).all()
            q = gmc.preference_loss(y, l2)
            assert torch.isnan(q[0]) and torch.isnan(q[3][1, 4])


def test_losses_without_tokens():
    import paper_1905_12948_amd as gmc
    x = torch.full((4, 3, 50), math.nan, device="cuda:0")
    labels = torch.full((4, 3), ref.IGNORE, device="cuda:0")
    for reduction in ("token", "sequence"):
        stats, logp, grad = gmc.policy_loss(x, labels, None, torch.ones(4, device="cuda:0"), reduction=reduction)
        assert not stats.any() and not logp.any() and not grad.any()
    for average in (False, True):
        loss, each, rewards, logp, grad = gmc.preference_loss(x, labels, average=average)
        assert torch.allclose(each, torch.full_like(each, math.log(2))) and abs(loss.item() - math.log(2)) < 1e-6
        assert not rewards.any() and not logp.any() and not grad.any()
    for shape in ((0, 3), (4, 0)):
        e = torch.zeros(*shape, 50, device="cuda:0")
        none = torch.zeros(shape, dtype=torch.int64, device="cuda:0")
        stats, _, grad = gmc.policy_loss(e, none, None, torch.ones(shape[0], device="cuda:0"))
        assert not stats.any() and grad.shape == e.shape
        loss = gmc.preference_loss(e, none)[0]
        assert abs(loss.item() - (math.log(2) if shape[0] else 0)) < 1e-6


def test_losses_far_offsets():
    """Sequences more than 2^32 elements apart."""
    for V in (100, 5000, 50257):
        big = torch.empty(2 ** 32 + 2 * V, device="cuda:0", dtype=torch.bfloat16)
        x = torch.randn(2, 2, V, device="cuda:0").bfloat16()
        v = big.as_strided((2, 2, V), (2 ** 32, V, 1))
        v.copy_(x)
        labels = torch.randint(0, V, (2, 2), device="cuda:0")
        # rows of another alignment are summed in another order: each result is within its own
        # bound of the truth (gradients: half a step and 2 LP of c p; all else: the log-probabilities')
        for a, b in zip(both_losses(v, labels), both_losses(x, labels)):
            if a.dtype == torch.bfloat16:
                torch.testing.assert_close(a, b, rtol=2 * (2.0 ** -9 + 2 * LP), atol=1e-10)
            else:
                torch.testing.assert_close(a, b, rtol=8 * U, atol=2 * (LP + 8 * U * 20))
        del big, v


def test_loss_gradients_against_differences():
    """The kernels' own losses at x +- h along directions; h^2 and the losses' 32-bit
    rounding over h bound the difference quotient's error."""
    import paper_1905_12948_amd as gmc
    torch.manual_seed(1)
    x = torch.randn(4, 6, 40, device="cuda:0")
    labels = torch.randint(0, 40, (4, 6), device="cuda:0")
    labels[0, :2] = ref.IGNORE
    adv = torch.tensor([1.0, -1.0, 2.0, -0.5], device="cuda:0")
    old, _, _ = gmc.policy_loss(x + 0.1 * torch.randn_like(x), labels, None, adv, grad=False)[1:] + (0,)
    refs = old + 0.1 * torch.randn_like(old)

    def policy(v, grad=True):
        s, _, g = gmc.policy_loss(v, labels, old, adv, ref_logp=refs, clip=(0.9, 5.0), kl_coef=0.3, grad=grad)
        return s[0].double(), g

    def preference(v, grad=True):
        out = gmc.preference_loss(v, labels, refs, beta=0.4, smoothing=0.05, grad=grad)
        return out[0].double(), out[4]

    h = 1e-2
    for f in (policy, preference):
        g = f(x)[1].double()
        for k in range(4):
            d = torch.randn(x.shape, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(k))
            quotient = (f(x + h * d, False)[0] - f(x - h * d, False)[0]) / (2 * h)
            # third derivatives along d of size at most about 30, losses of size about 3
            assert abs((quotient - (g * d.double()).sum()).item()) < 30 * h * h / 6 + 64 * U * 3 / h


def test_same_bits_streams_and_graphs():
    """Every operator twice, on a side stream, and in a captured graph that is replayed
    with other work between the replays: the same bits."""
    import paper_1905_12948_amd as gmc
    torch.manual_seed(3)
    x = torch.randn(6, 40, 40, 64, device="cuda:0").bfloat16()
    wide = torch.randn(2, 50, 50, 136, device="cuda:0")
    ga, be = torch.randn(64, device="cuda:0"), torch.randn(64, device="cuda:0")
    logits = torch.randn(4, 30, 5001, device="cuda:0").bfloat16()
    labels = torch.randint(0, 5001, (4, 30), device="cuda:0")
    labels[1, 20:] = ref.IGNORE

    def every():
        y, mean, rstd = gmc.group_norm(x, 8, ga, be, act="silu")
        z = gmc.dropout(y, 0.2, 4, t=2, worker=1, residual=x)
        dx = gmc.group_norm_backward(gmc.dropout_backward(z, 0.2, 4, t=2, worker=1), x, mean, rstd, ga, be, act="silu")
        w = gmc.group_norm(wide, 1, act="relu")
        dw = gmc.group_norm_backward(wide, wide, w[1], w[2], act="relu")
        return [y, mean, rstd, z, *dx, *w, *dw, *both_losses(logits, labels)]

    first = every()
    again = every()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        aside = every()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b, c in zip(first, again, aside):
        assert torch.equal(a, b) and torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = every()
    for k in range(4):
        for t in held:
            t.fill_(7)
        every()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(first, held):
            assert torch.equal(a, b), k


# -- many short rows: tokens, sequences and pairs counted by launches of their own ----


@pytest.mark.parametrize("R,T", [(2, 1500), (600, 3), (40, 60), (70, 1000)])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
def test_policy_loss_many_tokens(R, T, reduction):
    import paper_1905_12948_amd as gmc
    V = 20
    rng = np.random.default_rng(R)
    x = dev(2 * rng.normal(size=(R, T, V)))
    labels = rng.integers(0, V, (R, T))
    labels[rng.random((R, T)) < 0.3] = ref.IGNORE
    labels[::5] = ref.IGNORE
    adv = dev(rng.normal(size=R))
    y = np.maximum(labels, 0)
    table = ref.log_softmax(host(x))
    kept = labels != ref.IGNORE
    logp = np.where(kept, np.take_along_axis(table, y[:, :, None], 2)[:, :, 0], 0)
    old = dev(logp - rng.choice([-0.5, -0.1, 0.02, 0.4], (R, T)))
    A = host(adv)[:, None]
    ratio = np.exp(logp - host(old))
    free, bounded = ratio * A, np.clip(ratio, 0.8, 1.2) * A
    count = kept.sum(1, keepdims=True)
    weight = kept / (kept.sum() if reduction == "token" else np.maximum(count, 1) * (count > 0).sum())
    want = np.array([(weight * -np.minimum(free, bounded)).sum(), 0, (weight * (free > bounded)).sum()])
    c = weight * np.where(free <= bounded, -free, 0)
    grad = -c[:, :, None] * np.exp(table)
    np.put_along_axis(grad, y[:, :, None], np.take_along_axis(grad, y[:, :, None], 2) + c[:, :, None], 2)
    stats, lp, g = gmc.policy_loss(x, torch.as_tensor(labels).cuda(), old, adv, reduction=reduction)
    elp = np.where(kept, LP + 8 * U * np.abs(logp), 0.0)
    size = (weight * (elp + 16 * U) * ratio * np.abs(A)).sum()
    check(lp, logp, elp, "f32", "logp")
    check(stats, want, np.array([size + 8 * U * np.abs(want[0]), 0, 16 * U]), "f32", "stats")
    ec = weight * (elp + 16 * U) * 2 * ratio * np.abs(A)
    check(g, grad, logits_gradient_slack(c, ec, grad, labels, V), "f32", "gradient")


@pytest.mark.parametrize("P,T", [(2, 700), (9, 5), (400, 3), (3, 170), (3, 171), (8, 64), (8, 65)])
@pytest.mark.parametrize("average", [False, True])
def test_preference_loss_many_tokens(P, T, average):
    import paper_1905_12948_amd as gmc
    V, beta = 20, 0.1
    rng = np.random.default_rng(P)
    x = dev(2 * rng.normal(size=(2 * P, T, V)))
    labels = rng.integers(0, V, (2 * P, T))
    labels[rng.random((2 * P, T)) < 0.3] = ref.IGNORE
    labels[1] = ref.IGNORE
    loss, each, rewards, logp, c, grad = ref.preference(host(x), labels, None, beta, 0.1, average)
    got = gmc.preference_loss(x, torch.as_tensor(labels).cuda(), beta=beta, smoothing=0.1, average=average)
    kept = labels != ref.IGNORE
    elp = np.where(kept, LP + 8 * U * np.abs(logp), 0.0)
    share = 1 / np.maximum(kept.sum(1), 1) if average else np.ones(2 * P)
    er = beta * elp.sum(1) * share + U * np.abs(rewards)
    eh = er[:P] + er[P:]
    check(got[3], logp, elp, "f32", "logp")
    check(got[2], rewards, er, "f32", "rewards")
    check(got[1], each, eh + 4 * U * np.abs(each), "f32", "pair losses")
    check(got[0], loss, eh.mean() + 8 * U * abs(loss), "f32", "loss")
    ec = np.concatenate([eh, eh]) * beta * share / (4 * P) + 8 * U * np.abs(c)
    rows = np.ones((1, T))
    check(got[4], grad, logits_gradient_slack(c[:, None] * rows, ec[:, None] * rows, grad, labels, V), "f32", "gradient")
    alone = gmc.preference_loss(x, torch.as_tensor(labels).cuda(), beta=beta, smoothing=0.1, average=average, grad=False)
    assert torch.equal(alone[3], got[3])
    for a, b in zip(alone[:3], got[:3]):  # another order of the same 64-bit sums
        torch.testing.assert_close(a, b, rtol=4 * U, atol=1e-12)


@pytest.mark.parametrize("dtype,V", [("f32", 81920 + 13), ("f32", 120000), ("bf16", 163840 + 21), ("f16", 200001)])
def test_policy_loss_rows_read_twice(dtype, V):
    """Vocabularies that no workgroup's registers hold."""
    test_policy_loss(V, dtype)


@pytest.mark.parametrize("V", [120000, 170001])
def test_losses_over_logits_read_twice(V):
    test_losses_over_the_logits(V)


def test_rows_within_one_sum_range_or_shifted():
    """Logits around the ends of the range in which sums are taken unshifted: all
    near -28, near +41, one far above the others, and large negative levels."""
    import paper_1905_12948_amd as gmc
    rng = np.random.default_rng(4)
    for V in (17, 5000, 50257):
        rows = np.stack([rng.normal(size=V) + level for level in (-60, -29, -27, 0, 39, 42, 300, -3000)])
        rows[3, V // 2] = 45.0
        x = dev(rows[None])
        labels = torch.as_tensor(rng.integers(0, V, (1, len(rows)))).cuda()
        stats, logp, grad = gmc.policy_loss(x, labels, None, torch.ones(1, device="cuda:0"))
        _, _, _, lp, c, g = ref.policy(host(x), labels.cpu().numpy(), None, np.ones((1, len(rows))), None, 0.2, 0.2, 0, 1.0, False)
        # the exponent's argument is as large as the logits where they are not shifted: 2 u of 60 in
        # base 2 on top of the bounds above; x itself is exact
        elp = LP + 8 * U * np.abs(lp) + 120 * U
        check(logp, lp, elp, "f32", "logp")
        check(grad, g, logits_gradient_slack(c, np.abs(c) * 120 * U, g, labels.cpu().numpy(), V) * 1.5, "f32", "gradient")


def test_loss_gradients_take_the_logits_strides():
    """A nearly dense view's gradient has its strides, a sparse one's is contiguous;
    neither changes the values, and calls without the gradient give the same bits."""
    import paper_1905_12948_amd as gmc
    torch.manual_seed(6)
    full = torch.randn(4, 9, 5008, device="cuda:0").bfloat16()
    labels = torch.randint(0, 5000, (4, 8), device="cuda:0")
    labels[1, 3:] = ref.IGNORE
    adv = torch.randn(4, device="cuda:0")
    for v, like in ((full[:, :-1, :5000], True), (full[:, 1:, 3:5003], True), (full[:, :-1, :2000], False),
                    (full[:, ::2, :5000], False), (full[::2, :-1, :5000], False)):
        y = labels[:v.shape[0], :v.shape[1]].clamp(max=v.shape[2] - 1)
        a = adv[:v.shape[0]]
        for f in (lambda x, **k: gmc.policy_loss(x, y, None, a, **k), lambda x, **k: gmc.preference_loss(x, y, **k)):
            got, dense, alone = f(v), f(v.contiguous()), f(v, grad=False)
            assert got[-1].stride() == (v.stride() if like else v.contiguous().stride())
            for p, q in zip(alone[:-1], got[:-1]):
                assert torch.equal(p, q)
            # both within half a step, 2^-8, of the truth and 2 LP of c p
            torch.testing.assert_close(got[-1], dense[-1], rtol=2 * (2.0 ** -8 + 2 * LP), atol=1e-10)
            for p, q in zip(got[:-1], dense[:-1]):
                torch.testing.assert_close(p, q, rtol=8 * U, atol=8 * 2 * (LP + 8 * U * 20))
