"""The operators of a worker's forward and backward pass, as cases that can be
timed and compared: dropout with the residual add, group norm with its
activation (channels last), the preference loss and the clipped policy loss with
their gradients: what a worker runs between its data and the gradient that
gmc_step compresses.

A case is a dict of plain values:

  op       "dropout", "norm", "preference", "policy"
  dtype    the activations' or logits' type: "bf16", "f16", "f32"
  way      dropout, norm: "forward" or "backward" (the losses give loss and gradient)
  dropout  rows, cols; pitch: elements from one row to the next; p; add: with the residual
  norm     N images of H x W pixels with C channels in G groups; act
  losses   seqs sequences of T tokens with a vocabulary of V; pitch: elements from
           one token's logits to the next's; extra: tokens each sequence has beyond
           the T that count (a view without the last token); dirty: the ignored tokens'
           logits hold NaN and the vocabulary's last entries are -inf
  preference  seqs / 2 pairs; beta, smoothing, average (of the token log-probabilities)
  policy   lo, hi: the clip range; kl: its coefficient; tau: temperature; reduction
           "token" or "sequence"; scale: the gradient's scale (half precision)

With `own` false run() computes an operator from elementary torch operations in
32 bits, rounded once at the end; with `own` true it calls the framework.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
IGNORE = -100
LARGEST = 3.2e9              # bytes of the largest listed case, which a drawn one stays under

# the constants of SplitMix64 (Steele, Lea and Flood, OOPSLA 2014) as signed 64-bit numbers
GAMMA, MIX1, MIX2 = -7046029254386353131, -4658895280553007687, -7723592293110705685
MASK64 = (1 << 64) - 1


def _dropout(name, **c):
    return dict({"name": name, "op": "dropout", "dtype": "bf16", "way": "forward", "rows": 0, "cols": 768, "pitch": 768,
                 "p": 0.1, "add": True}, **c)


def _norm(name, **c):
    return dict({"name": name, "op": "norm", "dtype": "bf16", "way": "forward", "N": 1, "H": 7, "W": 7, "C": 64, "G": 32,
                 "act": "relu"}, **c)


def _preference(name, **c):
    return dict({"name": name, "op": "preference", "dtype": "bf16", "seqs": 2, "T": 16, "V": 50257, "pitch": 50257,
                 "extra": 0, "dirty": False, "beta": 0.1, "smoothing": 0.0, "average": False}, **c)


def _policy(name, **c):
    return dict({"name": name, "op": "policy", "dtype": "bf16", "seqs": 2, "T": 8, "V": 50257, "pitch": 50257, "extra": 0,
                 "dirty": False, "lo": 0.2, "hi": 0.2, "kl": 0.05, "tau": 1.0, "reduction": "token", "scale": 1.0}, **c)


def listed():
    return [
        # the smallest call: a few tokens of a 768-wide decoder, one residual branch
        _dropout("dropout few tokens", rows=16),
        # a decoder's batch of 16 sequences of 1024 tokens, its residual branch
        _dropout("dropout batch", rows=16384),
        # the gradient of a wide 32-bit activation whose rows are slices of a wider buffer, odd sizes
        _dropout("dropout backward odd", dtype="f32", way="backward", rows=8191, cols=1001, pitch=1024, p=0.5, add=False),
        # one image before a classifier's head: the last stage of an ImageNet ResNet-50
        _norm("norm one image", dtype="f32", C=2048, act="none"),
        # the first stage of a CIFAR ResNet-18, a worker's batch of 128
        _norm("norm cifar stage", N=128, H=32, W=32),
        # its gradient in the second stage
        _norm("norm cifar backward", way="backward", N=128, H=16, W=16, C=128),
        # the widest activations of an ImageNet ResNet-50 and the gradient, a worker's batch of 64
        _norm("norm imagenet stage", N=64, H=56, W=56, C=256, act="silu"),
        _norm("norm imagenet backward", way="backward", N=64, H=56, W=56, C=256),
        # one pair of short answers
        _preference("preference one pair"),
        # a worker's batch of pairs at a decoder's vocabulary, prompt and padding ignored
        _preference("preference batch", seqs=16, T=512, smoothing=0.1),
        # two short rollouts
        _policy("policy short"),
        # a worker's batch of rollouts: the largest
        _policy("policy batch", seqs=16, T=1024, extra=1),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    op = rng.choice(["dropout", "norm", "preference", "policy"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    way = rng.choice(["forward", "backward"])
    if op == "dropout":
        cols = rng.choice([64, 255, 768, 1001, 2048, 4096, _log(rng, 1, 9000)])
        rows = _log(rng, 1, 6e7 / cols)
        c = _dropout("", dtype=dtype, way=way, rows=rows, cols=cols, pitch=cols + rng.choice([0, 0, 1, 8, 24]),
                     p=rng.choice([0.0, 0.05, 0.1, 0.1, 0.3, 0.5]), add=way == "forward" and rng.random() < 0.6)
    elif op == "norm":
        G = rng.choice([1, 4, 8, 16, 32, 32, 32])
        C = G * rng.choice([1, 2, 3, 4, 8, 8, 16, 64])
        side = rng.choice([1, 4, 7, 8, 14, 16, 28, 32, 33, 56])
        if side * side * C < 32 * G:
            side = 7             # groups of a few values would give gradients that are all rounding
        W = rng.choice([side, side, max(1, side - 1)])
        N = _log(rng, 1, max(2, min(256, 5e7 / (C * side * W))))
        act = rng.choice(["none", "relu", "relu", "silu"])
        c = _norm("", dtype=dtype, way=way, N=N, H=side, W=W, C=C, G=G, act=act)
    else:
        V = rng.choice([17, 1000, 8191, 32000, 50257, 50257, 65536, 128001, _log(rng, 2, 150000)])
        T = _log(rng, 1, 1024)
        seqs = 2 * _log(rng, 1, max(2, min(24, 0.45 * LARGEST / (4 * V * T) / 2)))
        T = max(1, min(T, int(0.45 * LARGEST / (4 * V * seqs))))
        both = dict(dtype=dtype, seqs=seqs, T=T, V=V, pitch=V + rng.choice([0, 0, 7, (-V) % 64]), extra=rng.choice([0, 0, 1]),
                    dirty=V > 64 and rng.random() < 0.3)
        if op == "preference":
            c = _preference("", **both, smoothing=rng.choice([0.0, 0.0, 0.1]))
            c["average"] = rng.random() < 0.3
            c["beta"] = 2.0 if c["average"] else 0.1
        else:
            c = _policy("", **both, hi=rng.choice([0.2, 0.28]), kl=rng.choice([0.0, 0.02, 0.05]),
                        tau=rng.choice([1.0, 1.0, 0.7]), reduction=rng.choice(["token", "sequence"]))
            c["scale"] = 65536.0 if dtype == "f16" else 1.0
    del c["name"]
    return c


# -- what a user's program has in hand ------------------------------------


def _spans(seqs, T):
    """First and last + 1 of each sequence's tokens that count: a prompt of up to an eighth
    before them, and answers of a quarter of the length up to what the prompt leaves."""
    start = [int(T / 8 * (r * 0.381966 % 1)) for r in range(seqs)]
    return start, [a + max(1, math.ceil((T - a) * (0.25 + 0.75 * (0.5 + r * 0.618034) % 1))) if r != 5 else a
                   for r, a in enumerate(start)]


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _prepare_dropout(c, seed):
    g = _generator(seed)
    dtype = DTYPES[c["dtype"]]

    def rows():
        return _normal(g, c["rows"], c["pitch"]).to(dtype)[:, :c["cols"]]

    s = {"x": rows(), "seed": seed * 7919 + 12345, "t": 100 + seed % 1000, "worker": seed % 8, "site": seed % 24}
    s["residual"] = rows() if c["add"] else None
    return s


def _prepare_norm(c, seed):
    g = _generator(seed)
    dtype = DTYPES[c["dtype"]]
    # channels with levels and spreads of their own, as after a convolution
    x = _normal(g, c["N"], c["H"], c["W"], c["C"]) * torch.exp(0.5 * _normal(g, c["C"])) + 0.7 * _normal(g, c["C"])
    s = {"x": x.to(dtype), "gamma": 1 + 0.2 * _normal(g, c["C"]), "beta": 0.2 * _normal(g, c["C"]), "eps": 1e-5}
    if c["way"] == "backward":
        s["dy"] = _normal(g, c["N"], c["H"], c["W"], c["C"]).to(dtype)
        s["mean"], s["rstd"] = _moments(s["x"].float(), c["G"], s["eps"])
    return s


def _prepare_loss(c, seed):
    g = _generator(seed)
    seqs, T, V = c["seqs"], c["T"], c["V"]
    first, last = (torch.tensor(v, device=DEVICE)[:, None] for v in _spans(seqs, T))
    at = torch.arange(T, device=DEVICE)[None, :]
    kept = (at >= first) & (at < last)
    labels = torch.randint(0, max(1, V - 16 if c["dirty"] else V), (seqs, T), generator=g, device=DEVICE)
    data = torch.empty((seqs, T + c["extra"], c["pitch"]), dtype=DTYPES[c["dtype"]], device=DEVICE)
    sharp = 3.0 * math.sqrt(math.log(max(V, 3)) / 10.8)
    data.normal_(0.0, sharp, generator=g)
    logits = data[:, :T, :V]
    # a trained model gives its own tokens more than chance
    own_logit = (0.6 * sharp * math.sqrt(2 * math.log(max(V, 3))) + _normal(g, seqs, T)).to(logits.dtype)
    logits.scatter_(2, labels[:, :, None], own_logit[:, :, None])
    if c["dirty"]:
        logits[:, :, V - 16:] = -math.inf
        logits.masked_fill_(~kept[:, :, None], math.nan)
    labels = labels.masked_fill(~kept, IGNORE)
    s = {"logits": logits, "labels": labels}
    logp = _chosen(logits, labels.clamp(min=0), c.get("tau", 1.0))[0].masked_fill_(~kept, 0.0)
    if c["op"] == "preference":
        # the reference differs by a little at each token and by its taste for each answer
        taste = (0.5 if c["average"] else 8.0 / kept.sum(1, keepdim=True).clamp(min=1)) * _normal(g, seqs, 1)
        s["ref_logp"] = (logp + taste + 0.1 * _normal(g, seqs, T)).masked_fill_(~kept, 0.0)
        return s
    # the probability ratios of a few updates of the same rollouts, some beyond the clip
    # range; none within rounding of its ends, where the gradient jumps
    ratio = 0.15 * _normal(g, seqs, T)
    for end in (math.log1p(-c["lo"]), math.log1p(c["hi"])):
        ratio = torch.where((ratio - end).abs() < 2e-3, end + 4e-3, ratio)
    s["old_logp"] = (logp - ratio).masked_fill_(~kept, 0.0)
    s["ref_logp"] = (logp + 0.3 * _normal(g, seqs, T)).masked_fill_(~kept, 0.0) if c["kl"] else None
    s["advantages"] = _normal(g, seqs) + 0.3
    return s


def prepare(case, seed):
    make = {"dropout": _prepare_dropout, "norm": _prepare_norm}.get(case["op"], _prepare_loss)
    return dict(make(case, int(seed)), case=case)


# -- the plain forms --------------------------------------------------------


def _mix(z):
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * MIX1
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * MIX2
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _mix_int(z):
    z &= MASK64
    z = ((z ^ (z >> 30)) * (MIX1 & MASK64)) & MASK64
    z = ((z ^ (z >> 27)) * (MIX2 & MASK64)) & MASK64
    return z ^ (z >> 31)


def _stream(s):
    """The state of the mask's SplitMix64 stream: seed, step, worker and site."""
    z = s["seed"] ^ _mix_int(s["t"] + 1) ^ _mix_int((s["worker"] + 1) << 32 | (s["site"] + 1))
    return z & MASK64


def _signed(z):
    return z - (1 << 64) if z >> 63 else z


def _plain_dropout(c, s):
    x = s["x"].float()
    level = math.floor(c["p"] * 65536 + 0.5)
    # element i takes bits 16 (i mod 4) to 16 (i mod 4) + 15 of draw i // 4
    n = x.numel()
    draws = torch.arange(1, (n + 3) // 4 + 1, device=x.device) * GAMMA + _signed(_stream(s))
    part = torch.arange(0, 64, 16, device=x.device)
    bits = ((_mix(draws)[:, None] >> part) & 65535).reshape(-1)[:n].reshape(x.shape)
    y = torch.where(bits >= level, x * (65536.0 / (65536 - level)), torch.zeros_like(x))
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return y.to(s["x"].dtype)


def _grouped(x, G):
    return x.reshape(x.shape[0], -1, G, x.shape[-1] // G)


def _moments(x, G, eps):
    """Mean and reciprocal deviation of each image's groups, [N, G]."""
    x = _grouped(x, G)
    n = x.shape[1] * x.shape[3]
    mean = x.sum((1, 3)) / n
    centred = x - mean[:, None, :, None]
    return mean, 1.0 / torch.sqrt((centred * centred).sum((1, 3)) / n + eps)


def _normalised(x, mean, rstd, G):
    return ((_grouped(x, G) - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)


def _plain_norm(c, s):
    x, gamma, beta, G = s["x"].float(), s["gamma"], s["beta"], c["G"]
    forward = c["way"] == "forward"
    mean, rstd = _moments(x, G, s["eps"]) if forward else (s["mean"], s["rstd"])
    hat = _normalised(x, mean, rstd, G)
    z = hat * gamma + beta
    if forward:
        y = z.clamp(min=0) if c["act"] == "relu" else z / (1 + torch.exp(-z)) if c["act"] == "silu" else z
        return y.to(s["x"].dtype), mean, rstd
    dz = s["dy"].float()
    if c["act"] == "relu":
        dz = torch.where(z > 0, dz, torch.zeros_like(dz))
    elif c["act"] == "silu":
        gate = 1 / (1 + torch.exp(-z))
        dz = dz * (gate * (1 + z * (1 - gate)))
    n = x[0].numel() // G
    weighted = _grouped(dz * gamma, G)
    shared = _grouped(hat, G)
    s1 = weighted.sum((1, 3), keepdim=True) / n
    s2 = (weighted * shared).sum((1, 3), keepdim=True) / n
    dx = rstd[:, None, :, None] * (weighted - (s1 + shared * s2))
    return dx.reshape(x.shape).to(s["x"].dtype), (dz * hat).sum((0, 1, 2)), dz.sum((0, 1, 2))


def _chosen(logits, at, tau):
    """Log-probability of the entries `at` and all probabilities, from logits / tau."""
    x = logits.float()
    if tau != 1.0:
        x = x / tau
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    logp = torch.gather(x, -1, at[..., None]) - (top + torch.log(total))
    return logp[..., 0], e.div_(total)


def _gradient(p, at, kept, coef, dtype):
    """coef (one-hot - p) at the kept tokens, zero at the others."""
    coef = torch.where(kept, coef, torch.zeros_like(coef))[..., None]
    g = (p * -coef).masked_fill_(~kept[..., None], 0.0)
    return g.scatter_add_(-1, at[..., None], coef).to(dtype)


def _plain_preference(c, s):
    labels, P = s["labels"], c["seqs"] // 2
    kept = labels != IGNORE
    at = labels.clamp(min=0)
    logp, p = _chosen(s["logits"], at, 1.0)
    logp = torch.where(kept, logp, torch.zeros_like(logp))
    gain = c["beta"] * torch.where(kept, logp - s["ref_logp"], torch.zeros_like(logp)).sum(1)
    share = torch.ones_like(gain)
    if c["average"]:
        share = 1.0 / kept.sum(1).clamp(min=1)
        gain = gain * share
    h = gain[:P] - gain[P:]
    # -log sigmoid(h) and its mirror, neither of which overflows
    low = torch.log1p(torch.exp(-h.abs()))
    each = (1 - c["smoothing"]) * (low + (-h).clamp(min=0)) + c["smoothing"] * (low + h.clamp(min=0))
    slope = c["beta"] * (1 / (1 + torch.exp(-h)) - (1 - c["smoothing"])) / P
    coef = torch.cat([slope, -slope]) * share
    grad = _gradient(p, at, kept, coef[:, None].expand_as(logp), s["logits"].dtype)
    return each.sum() / P, each, gain, logp, grad


def _plain_policy(c, s):
    labels = s["labels"]
    kept = labels != IGNORE
    at = labels.clamp(min=0)
    logp, p = _chosen(s["logits"], at, c["tau"])
    logp = torch.where(kept, logp, torch.zeros_like(logp))
    count = kept.sum(1, keepdim=True)
    if c["reduction"] == "token":
        weight = kept / count.sum().clamp(min=1)
    else:
        weight = kept / count.clamp(min=1) / (count > 0).sum().clamp(min=1)
    ratio = torch.exp(logp - s["old_logp"])
    A = s["advantages"][:, None]
    free, bounded = ratio * A, ratio.clamp(1 - c["lo"], 1 + c["hi"]) * A
    slope = torch.where(free <= bounded, -free, torch.zeros_like(free))
    kl = torch.zeros_like(logp)
    if s["ref_logp"] is not None:
        d = s["ref_logp"] - logp
        kl = torch.exp(d) - d - 1
        slope = slope + c["kl"] * (1 - torch.exp(d))
    each = -torch.minimum(free, bounded) + c["kl"] * kl
    stats = torch.stack([(weight * each).sum(), (weight * kl).sum(), (weight * (free > bounded)).sum()])
    grad = _gradient(p, at, kept, c["scale"] / c["tau"] * weight * slope, s["logits"].dtype)
    return stats, logp, grad


def _own_run(c, s):
    import paper_1905_12948_amd as gmc
    if c["op"] == "dropout":
        where = dict(seed=s["seed"], t=s["t"], worker=s["worker"], site=s["site"])
        if c["way"] == "forward":
            return gmc.dropout(s["x"], c["p"], residual=s["residual"], **where)
        return gmc.dropout_backward(s["x"], c["p"], **where)
    if c["op"] == "norm":
        if c["way"] == "forward":
            return gmc.group_norm(s["x"], c["G"], s["gamma"], s["beta"], eps=s["eps"], act=c["act"])
        return gmc.group_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["beta"], act=c["act"])
    if c["op"] == "preference":
        return gmc.preference_loss(s["logits"], s["labels"], s["ref_logp"], beta=c["beta"], smoothing=c["smoothing"],
                                   average=c["average"], ignore=IGNORE)
    return gmc.policy_loss(s["logits"], s["labels"], s["old_logp"], s["advantages"], ref_logp=s["ref_logp"],
                           clip=(c["lo"], c["hi"]), kl_coef=c["kl"], temperature=c["tau"], reduction=c["reduction"],
                           ignore=IGNORE, grad_scale=c["scale"])


def run(state):
    """One pass.  dropout: y or dx; norm: y, mean, rstd or dx, dgamma, dbeta; preference:
    loss, each pair's loss, each sequence's implicit reward, the tokens' log-probabilities, the
    logits' gradient; policy: (loss, mean KL, clipped share), the tokens' log-probabilities,
    the logits' gradient."""
    c = state["case"]
    if own:
        return _own_run(c, state)
    plain = {"dropout": _plain_dropout, "norm": _plain_norm, "preference": _plain_preference, "policy": _plain_policy}
    return plain[c["op"]](c, state)


def work(case):
    c, b = case, SIZE[case["dtype"]]
    if c["op"] == "dropout":
        n = c["rows"] * c["cols"]
        return {"bytes": n * b * (3 if c["add"] else 2), "flops": n * (2 if c["add"] else 1)}
    if c["op"] == "norm":
        n = c["N"] * c["H"] * c["W"] * c["C"]
        forward = c["way"] == "forward"
        return {"bytes": n * b * (2 if forward else 3) + 8 * c["N"] * c["G"] + (8 if forward else 16) * c["C"],
                "flops": n * (8 if forward else 16)}
    first, last = _spans(c["seqs"], c["T"])
    kept, tokens = sum(z - a for a, z in zip(first, last)), c["seqs"] * c["T"]
    # the kept tokens' logits in, every token's gradient out
    return {"bytes": (kept + tokens) * c["V"] * b + tokens * 20, "flops": kept * c["V"] * 6}


# -- in 64 bits, from the definitions ---------------------------------------


def _exact_dropout(c, s):
    x = s["x"].double().cpu().numpy()
    if x.size > 60_000_000:
        return None
    n = x.size
    with np.errstate(over="ignore"):
        z = np.uint64(_stream(s)) + (np.arange(n, dtype=np.uint64) // np.uint64(4) + np.uint64(1)) * np.uint64(GAMMA & MASK64)
        for shift, factor in ((30, MIX1), (27, MIX2)):
            z = (z ^ (z >> np.uint64(shift))) * np.uint64(factor & MASK64)
    z ^= z >> np.uint64(31)
    z = (z >> (np.uint64(16) * (np.arange(n, dtype=np.uint64) % np.uint64(4)))) & np.uint64(65535)
    level = int(c["p"] * 65536 + 0.5)
    y = x * (z.reshape(x.shape) >= level) * 65536.0 / (65536.0 - level)
    if c["add"]:
        y += s["residual"].double().cpu().numpy()
    return y


def _exact_norm(c, s):
    N, C, G = c["N"], c["C"], c["G"]
    x = s["x"].double().view(N, -1, G, C // G)
    gamma, beta = s["gamma"].double().view(G, -1), s["beta"].double().view(G, -1)
    if c["way"] == "forward":
        var, mean = torch.var_mean(x, dim=(1, 3), correction=0, keepdim=True)
        rstd = (var + s["eps"]).rsqrt()
    else:
        mean, rstd = s["mean"].double().view(N, 1, G, 1), s["rstd"].double().view(N, 1, G, 1)
    hat = (x - mean) * rstd
    z = hat * gamma + beta
    if c["way"] == "forward":
        y = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v)}[c["act"]](z)
        return y.view(s["x"].shape), mean.view(N, G), rstd.view(N, G)
    dz = s["dy"].double().view(x.shape)
    if c["act"] == "relu":
        dz = dz * (z > 0)
    elif c["act"] == "silu":
        gate = torch.sigmoid(z)
        dz = dz * gate * (1 + z - z * gate)
    dgamma, dbeta = (dz * hat).sum((0, 1)).view(-1), dz.sum((0, 1)).view(-1)
    dhat = dz * gamma
    dx = rstd * (dhat - dhat.mean((1, 3), keepdim=True) - hat * (dhat * hat).mean((1, 3), keepdim=True))
    return dx.view(s["x"].shape), dgamma, dbeta


def _exact_tokens(s, tau):
    """The kept tokens (flat positions), their labels, log-probabilities and log-softmax rows."""
    labels = s["labels"].reshape(-1)
    rows = (labels != IGNORE).nonzero()[:, 0]
    T = s["labels"].shape[1]
    table = torch.log_softmax(s["logits"][rows // T, rows % T].double() / tau, -1)
    y = labels[rows]
    logp = torch.zeros(labels.shape, dtype=torch.float64, device=labels.device)
    logp[rows] = table[torch.arange(len(rows), device=rows.device), y]
    return rows, y, logp.view(s["labels"].shape), table


def _exact_grad(s, rows, y, table, coef):
    grad = torch.zeros((s["labels"].numel(), table.shape[1]), dtype=torch.float64, device=table.device)
    table.exp_().neg_()
    table[torch.arange(len(rows), device=rows.device), y] += 1
    grad[rows] = table * coef.reshape(-1)[rows][:, None]
    return grad.view(*s["labels"].shape, -1)


def _exact_preference(c, s):
    P = c["seqs"] // 2
    rows, y, logp, table = _exact_tokens(s, 1.0)
    length = (s["labels"] != IGNORE).sum(1).clamp(min=1).double()
    gain = c["beta"] * (logp.sum(1) - s["ref_logp"].double().sum(1)) / (length if c["average"] else 1.0)
    h = gain[:P] - gain[P:]
    each = -((1 - c["smoothing"]) * torch.nn.functional.logsigmoid(h) + c["smoothing"] * torch.nn.functional.logsigmoid(-h))
    dh = (c["smoothing"] * torch.sigmoid(h) - (1 - c["smoothing"]) * torch.sigmoid(-h)) * c["beta"] / P
    coef = torch.cat([dh, -dh]) / (length if c["average"] else 1.0)
    return each.mean(), each, gain, logp, _exact_grad(s, rows, y, table, coef[:, None].expand_as(logp))


def _exact_policy(c, s):
    rows, y, logp, table = _exact_tokens(s, c["tau"])
    kept = (s["labels"] != IGNORE).double()
    length = kept.sum(1, keepdim=True)
    weight = kept / kept.sum() if c["reduction"] == "token" else kept / length.clamp(min=1) / (length > 0).sum()
    ratio = (logp - s["old_logp"].double()).exp()
    A = s["advantages"].double()[:, None].expand_as(ratio)
    over = torch.where(A >= 0, ratio > 1 + c["hi"], ratio < 1 - c["lo"])
    edge = torch.where(A >= 0, 1 + c["hi"], 1 - c["lo"])
    loss, slope = -torch.where(over, edge, ratio) * A, torch.where(over, 0.0, -ratio * A)
    kl = torch.zeros_like(logp)
    if s["ref_logp"] is not None:
        d = s["ref_logp"].double() - logp
        kl = torch.expm1(d) - d
        slope = slope - c["kl"] * torch.expm1(d)
    stats = torch.stack([(weight * v).sum() for v in (loss + c["kl"] * kl, kl, over.double())])
    return stats, logp, _exact_grad(s, rows, y, table, weight * slope * c["scale"] / c["tau"])


def exact(case, seed):
    s = prepare(case, seed)
    made = {"dropout": _exact_dropout, "norm": _exact_norm, "preference": _exact_preference, "policy": _exact_policy}
    return made[case["op"]](case, s)
