"""Tokens' scores and orthogonalised matrices from their definitions, in 64 bits
(numpy): what gmc_token_scores, gmc_token_scores_backward, gmc_orthogonalize and
gmc_orthogonal_step are held against.  Shares no code with the library."""
import numpy as np

IGNORE = -100
QUINTIC = (3.4445, -4.7750, 2.0315)


def log_softmax(x, tau):
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        z = (x - x.max(-1, keepdims=True)) / tau
        return z - np.log(np.exp(z).sum(-1, keepdims=True))


def scores(x, tau, top):
    """(log-probabilities, entropy, mean of z^2, the places of the `top` largest) of rows x."""
    table = log_softmax(x, tau)
    with np.errstate(invalid="ignore"):
        p = np.exp(table)
        entropy = -np.where(p > 0, p * table, 0.0).sum(-1)
        z = table - table.max(-1, keepdims=True)
        spread = np.where(p > 0, p * z * z, 0.0).sum(-1)
    # NaN above all, then by value, equal ones by place
    key = np.where(np.isnan(x), np.inf, x)
    nan = np.isnan(x)
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[-1]), x.shape), -key, ~nan), axis=-1)
    return table, entropy, spread, order[..., :top]


def scores_gradient(x, tau, labels, dlogp, dentropy, ids, dtop):
    """The gradient of sum dlogp logp + dentropy H + sum dtop logp[ids] in rows x (2-d); labels
    of -1: none."""
    table = log_softmax(x, tau)
    p = np.exp(table)
    down = np.zeros_like(table)
    for r in range(len(x)):
        if labels[r] >= 0:
            down[r, labels[r]] += dlogp[r]
        for j, g in zip(ids[r], dtop[r]):
            if 0 <= j < x.shape[1]:
                down[r, j] += g
    share = np.where(p > 0, p * table, 0.0)
    down -= dentropy[:, None] * (p + share)
    return (down - p * down.sum(-1, keepdims=True)) / tau


def polar(x, steps=5, coefficients=QUINTIC, eps=1e-7, keep=lambda v: v):
    """The Newton-Schulz steps on x / (|x| + eps); keep: what becomes of each value that is kept."""
    x = np.asarray(x, np.float64)
    norm = np.sqrt((x * x).sum()) + eps
    x = keep(x / norm if norm > 0 else x)
    for k in range(steps):
        a, b, c = coefficients if np.ndim(coefficients) == 1 else coefficients[k]
        gram = keep(x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x)
        poly = keep(b * gram + c * (gram @ gram))
        x = keep(a * x + (poly @ x if x.shape[0] <= x.shape[1] else x @ poly))
    return x


def polar_spread(x, error, **how):
    """The largest of eight distances between the steps' result and theirs with values off by up to
    `error` of each, at random."""
    rng = np.random.default_rng(5)
    exact = polar(x, **how)
    noisy = [polar(x, keep=lambda v: v * (1 + error * rng.uniform(-1, 1, v.shape)), **how) for _ in range(8)]
    return max(np.linalg.norm(v - exact) for v in noisy)
