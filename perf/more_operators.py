"""Operators around a worker's loss and the server's update, as cases that can be
timed and compared: the scores of tokens (log-probabilities of given tokens, the
entropy of their distributions and the most probable alternatives) with the logits'
gradient, and the orthogonalisation of the matrices in a flat vector of parameters
by Newton-Schulz products, alone and as the server's step with its momentum.

A case is a dict of plain values:

  op       "scores", "scores_grad", "orth", "step"
  dtype    the logits', the vector's or the update's type: "bf16", "f16", "f32"
  scores   seqs sequences of T tokens with a vocabulary of V; pitch: elements from
           one token's logits to the next's; extra: tokens each sequence has beyond
           the T (a view without the last token); dirty: the ignored tokens' logits hold
           NaN and the vocabulary's last entries are -inf; labels: whether tokens are
           given (without them all tokens count); top: alternatives; tau: temperature
  scores_grad  the same, with gradients of the log-probabilities, of the entropies
           (entropy) and of the alternatives' log-probabilities (top)
  orth     table: which matrices the vector holds ("one": `count` of rows x cols, one
           after the other; "columns": `count` side by side, column slices of one wide
           array; "resnet18", "resnet50": those models' tensors); alpha
  step     the same, with mu, nesterov and decay; the server's update is sparse, as K
           workers' messages leave it

With `own` false run() computes an operator from elementary torch operations in
32 bits, rounded once at the end; with `own` true it calls the framework.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
IGNORE = -100
LARGEST = 1.7e9              # bytes of logits of the largest listed case
LARGEST_FLOPS = 1.4e12       # and operations of the largest orthogonalisation

STEPS, EPS = 5, 1e-7
A, B, C = 3.4445, -4.7750, 2.0315   # X <- A X + B (X X^T) X + C (X X^T)^2 X


def _scores(name, **c):
    return dict({"name": name, "op": "scores", "dtype": "bf16", "seqs": 1, "T": 1, "V": 50257, "pitch": 50257, "extra": 0,
                 "dirty": False, "labels": True, "top": 0, "tau": 1.0}, **c)


def _scores_grad(name, **c):
    return dict(_scores(name, op="scores_grad"), **dict({"entropy": True}, **c))


def _orth(name, **c):
    return dict({"name": name, "op": "orth", "dtype": "f32", "table": "one", "count": 1, "rows": 64, "cols": 64,
                 "alpha": 1.0}, **c)


def _step(name, **c):
    return dict(_orth(name, op="step"), **dict({"mu": 0.95, "nesterov": True, "decay": 0.0}, **c))


def listed():
    return [
        # a token just decoded, of one sequence: its distribution's entropy and five alternatives
        _scores("scores one token", labels=False, top=5),
        # the tokens that 64 sequences sampled in one step, with twenty alternatives
        _scores("scores decode step", dtype="f32", seqs=64, top=20, tau=0.8),
        # a worker's batch of rollouts before its policy loss: log-probabilities and entropies
        _scores("scores rollouts", seqs=16, T=1024, extra=1),
        # a batch of odd sizes with prompts and padding ignored and a part of the vocabulary masked
        _scores("scores odd", dtype="f16", seqs=6, T=333, V=32003, pitch=32064, extra=1, dirty=True, top=8, tau=0.7),
        # the gradient of a worker's batch, log-probabilities and an entropy bonus
        _scores_grad("scores gradient", seqs=16, T=512),
        # the gradient for a few teacher's alternatives as well, odd sizes in 32 bits
        _scores_grad("scores gradient odd", dtype="f32", seqs=4, T=129, V=8191, pitch=8200, top=5, dirty=True),
        # one small matrix: the stem of an ImageNet ResNet-50
        _orth("orth stem", rows=64, cols=147),
        # every matrix of a CIFAR ResNet-18's update
        _orth("orth resnet18", table="resnet18"),
        # one wide layer, the update in 16 bits
        _orth("orth wide layer", dtype="bf16", rows=2048, cols=2048),
        # the largest: one layer of 4096 x 4096 parameters
        _orth("orth large", rows=4096, cols=4096),
        # a 768-wide decoder's projections to queries, keys and values: column slices of one array
        _step("step projections", table="columns", count=3, rows=768, cols=768, decay=0.001),
        # every matrix of an ImageNet ResNet-50, the server's step
        _step("step resnet50", table="resnet50"),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    op = rng.choice(["scores", "scores", "scores_grad", "orth", "orth", "step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32", "f32"])
    if op in ("scores", "scores_grad"):
        V = rng.choice([17, 1000, 8191, 32000, 50257, 50257, 65536, 128001, _log(rng, 2, 200000)])
        part = (1.0 if op == "scores" else 0.5) * LARGEST / (4 * V)
        T = rng.choice([1, _log(rng, 1, 1024)])
        seqs = _log(rng, 1, max(2, min(96, part / T)))
        T = max(1, min(T, int(part / seqs)))
        both = dict(dtype=dtype, seqs=seqs, T=T, V=V, pitch=V + rng.choice([0, 0, 7, (-V) % 64]), extra=rng.choice([0, 0, 1]),
                    dirty=V > 64 and rng.random() < 0.3, tau=rng.choice([1.0, 1.0, 0.7]),
                    top=min(V, rng.choice([0, 0, 1, 5, 8, 20, 32])))
        if op == "scores":
            c = _scores("", **both)
            c["labels"] = rng.random() < 0.8
        else:
            c = _scores_grad("", **both)
            c["entropy"] = rng.random() < 0.7
    else:
        table = rng.choice(["one", "one", "one", "columns", "columns", "resnet18", "resnet50"])
        if op == "orth" and table == "resnet50":
            table = "one"
        c = (_orth if op == "orth" else _step)("", dtype=dtype, table=table)
        if table in ("one", "columns"):
            while True:
                c["rows"], c["cols"] = (rng.choice([64, 100, 256, 768, 1024, 2047, _log(rng, 1, 4096), _log(rng, 1, 4096)])
                                        for _ in range(2))
                c["count"] = _log(rng, 1, 24)
                if work(c)["flops"] < 0.8 * LARGEST_FLOPS and c["count"] * c["rows"] * c["cols"] < 2.5e7:
                    break
        if op == "orth":
            c["alpha"] = rng.choice([1.0, 0.02])
        else:
            c["nesterov"], c["decay"] = rng.random() < 0.7, rng.choice([0.0, 0.0, 0.002])
    del c["name"]
    return c


# -- the matrices of a flat vector ----------------------------------------------


def _resnet18():
    """CIFAR ResNet-18, a convolution as output channels x (input channels, window); 1 row: a norm's vectors."""
    s, cin = [(64, 27), (1, 128)], 64
    for stage, w in enumerate([64, 128, 256, 512]):
        for b in range(2):
            s += [(w, 9 * cin), (1, 2 * w), (w, 9 * w), (1, 2 * w)]
            if b == 0 and stage > 0:
                s += [(w, cin), (1, 2 * w)]
            cin = w
    return s + [(10, 512), (1, 10)]


def _resnet50():
    """ImageNet ResNet-50: 7x7 stem, bottlenecks [3, 4, 6, 3], 1000 classes."""
    s, cin = [(64, 147), (1, 128)], 64
    for blocks, w in zip([3, 4, 6, 3], [64, 128, 256, 512]):
        for b in range(blocks):
            s += [(w, cin), (1, 2 * w), (w, 9 * w), (1, 2 * w), (4 * w, w), (1, 8 * w)]
            if b == 0:
                s += [(4 * w, cin), (1, 8 * w)]
            cin = 4 * w
    return s + [(1000, 2048), (1, 1000)]


def _layout(c):
    """(components of the vector, its matrices as (offset, rows, cols, pitch))."""
    if c["table"] == "columns":
        wide = c["count"] * c["cols"]
        return c["rows"] * wide, [(k * c["cols"], c["rows"], c["cols"], wide) for k in range(c["count"])]
    tensors = {"resnet18": _resnet18, "resnet50": _resnet50}.get(c["table"], lambda: [(c["rows"], c["cols"])] * c["count"])()
    at, matrices = 0, []
    for m, n in tensors:
        if m > 1 or c["table"] == "one":
            matrices.append((at, m, n, n))
        at += m * n
    return at, matrices


def _view(x, matrix):
    at, m, n, pitch = matrix
    return torch.as_strided(x, (m, n), (pitch, 1), x.storage_offset() + at)


# -- what a user's program has in hand ------------------------------------------


def _spans(c):
    """First and last + 1 of each sequence's tokens that count: a prompt of up to an eighth
    before them, and answers of a quarter of the length up to what the prompt leaves."""
    seqs, T = c["seqs"], c["T"]
    if not c["labels"] or T == 1:
        return [0] * seqs, [T] * seqs
    start = [int(T / 8 * (r * 0.381966 % 1)) for r in range(seqs)]
    return start, [a + max(1, math.ceil((T - a) * (0.25 + 0.75 * (0.5 + r * 0.618034) % 1))) if r != 5 else a
                   for r, a in enumerate(start)]


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _prepare_scores(c, seed):
    g = _generator(seed)
    seqs, T, V = c["seqs"], c["T"], c["V"]
    first, last = (torch.tensor(v, device=DEVICE)[:, None] for v in _spans(c))
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
    s = {"logits": logits, "labels": labels.masked_fill(~kept, IGNORE) if c["labels"] else None}
    if c["op"] == "scores_grad":
        # what the forward call left, and what the program that takes its results gives back
        _, s["entropy"], _, s["top_ids"], s["norm"] = _plain_scores(c, s)
        s["dlogp"] = _normal(g, seqs, T) / (seqs * T)
        s["dentropy"] = 0.01 * (1 + _normal(g, seqs, T).abs()) / (seqs * T) if c["entropy"] else None
        s["dtop"] = _normal(g, seqs, T, c["top"]) / (seqs * T) if c["top"] else None
    return s


def _prepare_matrices(c, seed):
    g = _generator(seed)
    d, matrices = _layout(c)
    x = _normal(g, d) * 1e-4
    for m in matrices:
        # a gradient's matrix: a few strong directions over noise, at the layer's own size
        _, rows, cols, _ = m
        rank = max(1, min(8, rows // 2, cols // 2))
        strong = _normal(g, rows, rank) @ (_normal(g, rank, cols) / math.sqrt(rank))
        size = 10.0 ** (-2 - 2 * torch.rand(1, generator=g, device=DEVICE))
        _view(x, m).copy_((0.5 * strong + _normal(g, rows, cols)) * size)
    s = {"d": d, "matrices": matrices}
    if c["op"] == "orth":
        s["x"] = x.to(DTYPES[c["dtype"]])
    else:
        # the momentum is the past's; of the update two in a hundred components were sent
        s["momentum"] = x
        s["w"] = 0.02 * _normal(g, d)
        sent = torch.rand(d, generator=g, device=DEVICE) < 0.02
        s["update"] = (_normal(g, d) * x.abs() * sent).to(DTYPES[c["dtype"]])
        s["next"] = torch.empty(d, device=DEVICE)
    if own:
        import paper_1905_12948_amd as gmc
        s["plan"] = gmc.Matrices(d, matrices, scales=[_shape_scale(m) for m in matrices], device=DEVICE)
    return s


def _shape_scale(matrix):
    """The factor of a matrix's step: tall ones take longer ones."""
    return math.sqrt(max(1.0, matrix[1] / matrix[2]))


def prepare(case, seed):
    make = _prepare_scores if case["op"].startswith("scores") else _prepare_matrices
    return dict(make(case, int(seed)), case=case)


# -- the plain forms --------------------------------------------------------------


def _masked(v, kept, fill=0):
    return v if kept is None else v.masked_fill_(~kept.reshape(kept.shape + (1,) * (v.dim() - 2)), fill)


def _order(x):
    """64-bit keys of x's entries along the last axis that sort by value and, among equals, by place, the first highest."""
    bits = (x + 0.0).view(torch.int32).to(torch.int64)
    key = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    return (key << 32) - torch.arange(x.shape[-1], device=x.device)


def _plain_scores(c, s):
    logits, labels, tau = s["logits"].float(), s["labels"], c["tau"]
    kept = None if labels is None else labels != IGNORE
    top = logits.amax(-1, keepdim=True)
    z = (logits - top) / tau
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    log_total = torch.log(total)
    # sum of p (-log p), where p is 0 without a share
    entropy = (log_total - torch.where(e > 0, e * z, torch.zeros_like(e)).sum(-1, keepdim=True) / total)[..., 0]
    logp = None
    if labels is not None:
        logp = _masked((torch.gather(z, -1, labels.clamp(min=0)[..., None]) - log_total)[..., 0], kept)
    top_logp = top_ids = None
    if c["top"]:
        top_ids = torch.topk(_order(logits), c["top"], dim=-1).indices
        top_logp = _masked(torch.gather(z, -1, top_ids) - log_total, kept)
        top_ids = _masked(top_ids, kept, -1)
    norm = _masked(torch.cat([top, log_total], -1), kept)
    return logp, _masked(entropy, kept), top_logp, top_ids, norm


def _plain_scores_grad(c, s):
    logits, labels, norm = s["logits"].float(), s["labels"], s["norm"]
    kept = None if labels is None else labels != IGNORE
    logq = (logits - norm[..., :1]) / c["tau"] - norm[..., 1:]
    p = torch.exp(logq)
    direct = s["dlogp"].clone()
    if s["dtop"] is not None:
        direct += s["dtop"].sum(-1)
    slope = -direct[..., None]
    if s["dentropy"] is not None:
        slope = slope - s["dentropy"][..., None] * torch.where(p > 0, logq + s["entropy"][..., None], torch.zeros_like(p))
    grad = p * slope
    grad.scatter_add_(-1, labels.clamp(min=0)[..., None], s["dlogp"][..., None])
    if s["dtop"] is not None:
        grad.scatter_add_(-1, s["top_ids"].clamp(min=0), s["dtop"])
    return _masked(grad / c["tau"], kept).to(s["logits"].dtype)


def _orthogonalised(x):
    """Newton-Schulz steps on x over its Frobenius norm."""
    wide = x if x.shape[0] <= x.shape[1] else x.T
    wide = wide / (torch.sqrt((wide.double() * wide.double()).sum()).float() + EPS)
    for _ in range(STEPS):
        gram = wide @ wide.T
        wide = A * wide + (B * gram + C * (gram @ gram)) @ wide
    return wide if x.shape[0] <= x.shape[1] else wide.T


def _plain_orth(c, s):
    x = s["x"].float()
    out = x.clone()
    for m in s["matrices"]:
        _view(out, m).copy_(c["alpha"] * _shape_scale(m) * _orthogonalised(_view(x, m)))
    return out.to(s["x"].dtype)


RATE = 0.02


def _plain_step(c, s):
    w, momentum, update = s["w"], s["momentum"], s["update"].float()
    out = torch.add(w, update, out=s["next"])
    for m in s["matrices"]:
        u, v = _view(update, m), _view(momentum, m)
        v.copy_(c["mu"] * v + u)
        u = u + c["mu"] * v if c["nesterov"] else v
        _view(out, m).copy_((1 - c["decay"]) * _view(w, m) + RATE * _shape_scale(m) * _orthogonalised(u))
    return out, momentum


def _own_run(c, s):
    import paper_1905_12948_amd as gmc
    if c["op"] == "scores":
        return gmc.token_scores(s["logits"], s["labels"], top=c["top"], temperature=c["tau"], ignore=IGNORE)
    if c["op"] == "scores_grad":
        return gmc.token_scores_backward(s["logits"], s["norm"], s["labels"], dlogp=s["dlogp"], entropy=s["entropy"],
                                         dentropy=s["dentropy"], top_ids=s["top_ids"], dtop=s["dtop"],
                                         temperature=c["tau"], ignore=IGNORE)
    how = dict(steps=STEPS, coefficients=(A, B, C), eps=EPS)
    if c["op"] == "orth":
        return gmc.orthogonalize(s["plan"], s["x"], alpha=c["alpha"], **how)
    gmc.orthogonal_step(s["plan"], s["w"], s["update"], s["momentum"], RATE, mu=c["mu"], nesterov=c["nesterov"],
                        decay=c["decay"], w_out=s["next"], **how)
    return s["next"], s["momentum"]


def run(state):
    """One pass.  scores: the tokens' log-probabilities, the entropies, the alternatives'
    log-probabilities and places, and (largest logit, log of the sum over exp of the others'
    distances to it); scores_grad: the logits' gradient; orth: the vector with its matrices
    orthogonalised; step: the new parameters and the momentum."""
    c = state["case"]
    if own:
        return _own_run(c, state)
    plain = {"scores": _plain_scores, "scores_grad": _plain_scores_grad, "orth": _plain_orth, "step": _plain_step}
    return plain[c["op"]](c, state)


def work(case):
    c, b = case, SIZE[case["dtype"]]
    if c["op"] in ("scores", "scores_grad"):
        first, last = _spans(c)
        kept, tokens = sum(z - a for a, z in zip(first, last)), c["seqs"] * c["T"]
        if c["op"] == "scores":
            # the kept tokens' logits in; their scores and alternatives out
            return {"bytes": kept * c["V"] * b + tokens * (24 + 12 * c["top"]), "flops": kept * c["V"] * 8}
        # the kept tokens' logits in, every token's gradient out
        return {"bytes": (kept + tokens) * c["V"] * b + tokens * (28 + 12 * c["top"]), "flops": kept * c["V"] * 8}
    d, matrices = _layout(c)
    flops = 0
    for _, m, n, _ in matrices:
        m, n = min(m, n), max(m, n)
        # X X^T and its square are symmetric, half of each is enough; the product with X is whole
        flops += STEPS * (m * m * n + m * m * m + 2 * m * m * n)
    return {"bytes": d * (2 * b if c["op"] == "orth" else b + 16), "flops": flops}


# -- in 64 bits, from the definitions -----------------------------------------------


def _exact_rows(c, s):
    """The kept tokens' flat positions and their rows of log-probabilities."""
    seqs, T = c["seqs"], c["T"]
    if s["labels"] is None:
        rows = torch.arange(seqs * T, device=DEVICE)
    else:
        rows = (s["labels"].reshape(-1) != IGNORE).nonzero()[:, 0]
    x = s["logits"][rows // T, rows % T].double()
    return rows, x, torch.log_softmax(x / c["tau"], -1)


def _exact_scores(c, s):
    rows, x, table = _exact_rows(c, s)
    shape = (c["seqs"], c["T"])

    def spread(v, fill=0):
        out = torch.full((shape[0] * shape[1],) + v.shape[1:], fill, dtype=v.dtype, device=DEVICE)
        out[rows] = v
        return out.view(shape + v.shape[1:])

    logp = None
    if s["labels"] is not None:
        logp = spread(torch.take_along_dim(table, s["labels"].reshape(-1)[rows][:, None], 1)[:, 0])
    # -sum p log p: entr() is 0 at p = 0
    entropy = spread(torch.special.entr(table.exp()).sum(-1))
    top = x.max(-1).values
    norm = spread(torch.stack([top, torch.logsumexp((x - top[:, None]) / c["tau"], -1)], -1))
    top_logp = top_ids = None
    if c["top"]:
        ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
        top_logp, top_ids = spread(torch.take_along_dim(table, ids, 1)), spread(ids, -1)
    return logp, entropy, top_logp, top_ids, norm


def _exact_scores_grad(c, s):
    rows, x, table = _exact_rows(c, s)
    n, V = table.shape
    p = table.exp()
    down = torch.zeros(n, V, dtype=torch.float64, device=DEVICE)   # what each log-probability gets
    each = torch.arange(n, device=DEVICE)
    down[each, s["labels"].reshape(-1)[rows]] = s["dlogp"].reshape(-1)[rows].double()
    if s["dtop"] is not None:
        ids = s["top_ids"].reshape(-1, c["top"])[rows]
        down.index_put_((each[:, None].expand_as(ids), ids), s["dtop"].reshape(-1, c["top"])[rows].double(), accumulate=True)
    if s["dentropy"] is not None:
        # H = -sum p log p: its slope along log p_j is -p_j (1 + log p_j)
        down -= s["dentropy"].reshape(-1)[rows].double()[:, None] * (p + torch.where(p > 0, p * table, 0.0))
    grad = torch.zeros(c["seqs"] * c["T"], V, dtype=torch.float64, device=DEVICE)
    grad[rows] = (down - p * down.sum(-1, keepdim=True)) / c["tau"]
    return grad.view(c["seqs"], c["T"], V)


def _exact_polar(x):
    """The steps on x / (|x| + EPS), the products taken from the side of the shorter axis, one factor at a time."""
    x = x.double()
    x = x / (torch.linalg.matrix_norm(x) + EPS)
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            gram = x @ x.mT
            once = gram @ x
            x = A * x + B * once + C * (gram @ once)
        else:
            gram = x.mT @ x
            once = x @ gram
            x = A * x + B * once + C * (once @ gram)
    return x


def _exact_orth(c, s):
    out = s["x"].double()
    for at, m, n, pitch in s["matrices"]:
        here = out.as_strided((m, n), (pitch, 1), at)
        here.copy_(_exact_polar(here.clone()) * (c["alpha"] * math.sqrt(max(m, n) / n)))
    return out


def _exact_step(c, s):
    update, out = s["update"].double(), s["w"].double()
    momentum, before = s["momentum"].double(), s["w"].double()
    out += update
    for at, m, n, pitch in s["matrices"]:
        u, v, w, o = (t.as_strided((m, n), (pitch, 1), at) for t in (update, momentum, before, out))
        v.mul_(c["mu"]).add_(u)
        moved = _exact_polar(u + c["mu"] * v if c["nesterov"] else v)
        o.copy_(w - c["decay"] * w + (RATE * math.sqrt(max(m, n) / n)) * moved)
    return out, momentum


def exact(case, seed):
    s = prepare(case, seed)
    made = {"scores": _exact_scores, "scores_grad": _exact_scores_grad, "orth": _exact_orth, "step": _exact_step}
    return made[case["op"]](case, s)
