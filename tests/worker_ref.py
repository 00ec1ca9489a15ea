"""The worker-side operators from their definitions, in 64 bits on the CPU
(numpy): what the kernels of gmc_dropout, gmc_group_norm, gmc_policy_loss and
gmc_preference_loss are held against.  Shares no code with the library."""
import numpy as np

M64 = (1 << 64) - 1
IGNORE = -100


def mix(z):
    z &= M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def dropout_bits(index, seed, t, worker, site):
    """The 16 bits of the elements `index` (Python integers throughout)."""
    state = (seed ^ mix(t + 1) ^ mix(((worker + 1) << 32) | (site + 1))) & M64
    return np.array([(mix(state + (i // 4 + 1) * 0x9E3779B97F4A7C15) >> (16 * (i % 4))) & 0xFFFF
                     for i in map(int, index)], np.int64)


def dropout(x, p, seed, t, worker, site, residual=None, first=0):
    """y for elements first, first + 1, ... of a call."""
    x = np.asarray(x, np.float64)
    level = int(np.floor(65536 * p + 0.5))
    bits = dropout_bits(range(first, first + x.size), seed, t, worker, site).reshape(x.shape)
    keep = bits >= level
    scale = 65536.0 / (65536 - level) if level < 65536 else 0.0
    y = np.where(keep, x, 0.0) * scale
    return (y if residual is None else y + np.asarray(residual, np.float64)), keep


def act(z, kind):
    with np.errstate(over="ignore"):
        return {"none": z, "relu": np.maximum(z, 0), "silu": z / (1 + np.exp(-z))}[kind]


def act_slope(z, kind):
    with np.errstate(over="ignore"):
        g = 1 / (1 + np.exp(-z))
    return {"none": np.ones_like(z), "relu": (z > 0) * 1.0, "silu": g * (1 + z * (1 - g))}[kind]


def group_norm(x, G, gamma, beta, eps, kind, mean=None, rstd=None):
    """y, mean, rstd, hat, z of x [N, S, C]."""
    N, S, C = x.shape
    v = x.reshape(N, S, G, C // G)
    if mean is None:
        mean = v.mean((1, 3))
        rstd = 1 / np.sqrt(((v - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)
    hat = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, S, C)
    z = hat * gamma + beta
    return act(z, kind), mean, rstd, hat, z


def group_norm_backward(dy, x, G, gamma, beta, kind, mean, rstd):
    N, S, C = x.shape
    _, _, _, hat, z = group_norm(x, G, gamma, beta, 0.0, kind, mean, rstd)
    dz = dy * act_slope(z, kind)
    w, h = (dz * gamma).reshape(N, S, G, -1), hat.reshape(N, S, G, -1)
    m = S * (C // G)
    s1, s2 = w.sum((1, 3), keepdims=True), (w * h).sum((1, 3), keepdims=True)
    dx = rstd[:, None, :, None] * (w - (s1 + h * s2) / m)
    return dx.reshape(N, S, C), (dz * hat).sum((0, 1)), dz.sum((0, 1))


def log_softmax(x):
    top = x.max(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        # the difference first: at a top of -3e38 adding the logarithm to it would lose it
        return (x - top) - np.log(np.exp(x - top).sum(-1, keepdims=True))


def policy(logits, labels, old, adv, ref, lo, hi, kl_coef, tau, by_sequence):
    """loss, kl, clipped, logp, c (dloss/dlogp), gradient; adv [R, T]."""
    R, T, V = logits.shape
    kept = labels != IGNORE
    logp, grad, c = np.zeros((R, T)), np.zeros_like(logits), np.zeros((R, T))
    total, kls, clips = 0.0, 0.0, 0.0
    n = kept.sum()
    some = (kept.sum(1) > 0).sum()
    for r, t in zip(*np.nonzero(kept)):
        w = 1 / n if not by_sequence else 1 / (kept[r].sum() * some)
        table = log_softmax(logits[r, t] / tau)
        y = labels[r, t]
        lp = logp[r, t] = table[y]
        ratio = np.exp(lp - old[r, t]) if old is not None else 1.0
        A = adv[r, t]
        free, bounded = ratio * A, min(max(ratio, 1 - lo), 1 + hi) * A
        slope, loss, kl = (-free if free <= bounded else 0.0), -min(free, bounded), 0.0
        if ref is not None:
            d = ref[r, t] - lp
            kl = np.expm1(d) - d
            slope += kl_coef * (1 - np.exp(d))
        total += w * (loss + kl_coef * kl)
        kls += w * kl
        clips += w * (free > bounded)
        c[r, t] = w * slope
        onehot = np.zeros(V)
        onehot[y] = 1
        grad[r, t] = c[r, t] / tau * (onehot - np.exp(table))
    return total, kls, clips, logp, c, grad


def preference(logits, labels, ref, beta, smoothing, average):
    """loss, pair losses, rewards, logp, c, gradient."""
    R, T, V = logits.shape
    P = R // 2
    kept = labels != IGNORE
    logp, grad = np.zeros((R, T)), np.zeros_like(logits)
    tables = {}
    for r, t in zip(*np.nonzero(kept)):
        tables[r, t] = log_softmax(logits[r, t])
        logp[r, t] = tables[r, t][labels[r, t]]
    diff = np.where(kept, logp - (ref if ref is not None else 0.0), 0.0)
    share = 1 / np.maximum(kept.sum(1), 1) if average else np.ones(R)
    rewards = beta * diff.sum(1) * share
    h = rewards[:P] - rewards[P:]
    each = (1 - smoothing) * np.logaddexp(0, -h) + smoothing * np.logaddexp(0, h)
    dh = smoothing / (1 + np.exp(-h)) - (1 - smoothing) / (1 + np.exp(h))
    c = np.concatenate([dh, -dh]) * beta * share / P
    for (r, t), table in tables.items():
        onehot = np.zeros(V)
        onehot[labels[r, t]] = 1
        grad[r, t] = c[r] * (onehot - np.exp(table))
    return each.mean() if P else 0.0, each, rewards, logp, c, grad
