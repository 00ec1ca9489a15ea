"""The operators of a worker's own pass (include/gmc.h), on torch tensors:
dropout, group norm with its activation, the policy and preference losses
with their gradients, and tokens' scores (log-probabilities, entropies, the most
probable tokens) with theirs.

Like the rest of the binding this only marshals arguments: it checks types,
devices, shapes and strides, allocates outputs and scratch, and calls the
library on torch's current stream of the tensors' device.  There is no autograd
here: a backward call is a call, and a loss returns the logits' gradient
(``logits.backward(grad)`` carries it on).
"""
from __future__ import annotations

import math
from typing import Tuple

from .gmc import GMC_OK, GmcError, _raw_stream, _torch, load

ACTS = {"none": 0, "relu": 1, "silu": 2}
REDUCTIONS = {"token": 0, "sequence": 1}
IGNORE = -100

_codes = None

# As in gmc.py, the checks take the cheapest form of each test: at small sizes a
# call is bound by this code and its launches.


def _code(t, name: str) -> int:
    """The library's element type of t (float32, bfloat16 or float16, on a GPU)."""
    global _codes
    torch = _torch()
    if _codes is None:
        _codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    code = _codes.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float32, bfloat16 or float16, got %s" % (name, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be on a GPU device" % name)
    return code


def _int(v: int, bits: int, name: str) -> int:
    """v, an integer of the C interface, of which ctypes would take the low bits.  The
    callers look at its high bits first, which is the cheaper test."""
    if not -1 << (bits - 1) <= v < 1 << (bits - 1):
        raise ValueError("%s must be a %d-bit integer, got %d" % (name, bits, v))
    return v


def _is(t, dtype, shape, ref, name: str):
    """t is a tensor of a type and shape on ref's device."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.get_device() != ref.get_device():
        raise ValueError("%s must be on %s" % (name, ref.device))
    if t.shape != shape:
        raise ValueError("%s must have the shape %s, has %s" % (name, tuple(shape), tuple(t.shape)))


def _f32(t, shape, ref, name: str) -> int:
    """Pointer of a contiguous fp32 tensor of a shape, on ref's device (None: 0)."""
    if t is None:
        return 0
    _is(t, _torch().float32, shape, ref, name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def _new(ref, *shape):
    """A new fp32 tensor on ref's device."""
    return ref.new_empty(shape, dtype=_torch().float32)


def _another(t, ref, *shape):
    """A new fp32 tensor of a shape on ref's device; t, if there, is one such
    (taking its shape is the faster way)."""
    return _new(ref, *shape) if t is None else _torch().empty_like(t)


def _new_like(t):
    """A new contiguous tensor of t's shape and type."""
    torch = _torch()
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _call(t, entry, *args):
    """An entry point of the library on torch's current stream of t's device."""
    torch = _torch()
    dev = t.get_device()
    if dev == torch.cuda.current_device():
        st = entry(_raw_stream(t), *args)
    else:
        with torch.cuda.device(dev):
            st = entry(_raw_stream(t), *args)
    if st != GMC_OK:
        raise GmcError(st, load().gmc_last_error(None).decode())


def _rows(t, name: str) -> Tuple[int, int, int]:
    """(rows, cols, pitch) of a tensor whose last axis is contiguous and whose
    other axes are evenly spaced rows."""
    if t.dim() == 0:
        return 1, 1, 1
    cols = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols, cols
    if t.stride(-1) != 1 and cols > 1:
        raise ValueError("%s needs a contiguous last axis" % name)
    return t.numel() // cols, cols, _joined(t, t.dim() - 1, name)


def _joined(t, axes: int, name: str) -> int:
    """The one stride the first `axes` axes of t have as a single axis."""
    pitch, step = None, 0
    for k in range(axes - 1, -1, -1):
        if t.shape[k] == 1:
            continue
        if pitch is None:
            pitch = step = t.stride(k)
        elif t.stride(k) != step:
            raise ValueError("%s needs evenly spaced rows" % name)
        step *= t.shape[k]
    return t.shape[-1] if pitch is None else pitch


def dropout(x, p: float, seed: int, t: int = 0, worker: int = 0, site: int = 0, residual=None, out=None):
    """Dropout of x and, with ``residual``, the sum residual + dropout(x).  The
    mask is a function of (seed, t, worker, site) and the element's number in
    x.  ``out`` may be x or residual."""
    code = _code(x, "x")
    rows, cols, pitch = _rows(x, "x")
    pr = rp = 0
    if residual is not None:
        _is(residual, x.dtype, x.shape, x, "residual")
        rp = _rows(residual, "residual")[2]
        pr = residual.data_ptr()
    if out is None:
        out = _new_like(x)
        op = cols
    else:
        _is(out, x.dtype, x.shape, x, "out")
        op = _rows(out, "out")[2]
    t, worker, site = int(t), int(worker), int(site)
    if (t | worker | site) >> 31:
        _int(t, 64, "t"), _int(worker, 32, "worker"), _int(site, 32, "site")
    _call(x, load().gmc_dropout, code, rows, cols, x.data_ptr(), pitch, pr, rp, out.data_ptr(), op, float(p),
          int(seed) & (2 ** 64 - 1), t, worker, site)
    return out


def dropout_backward(dy, p: float, seed: int, t: int = 0, worker: int = 0, site: int = 0, out=None):
    """x's gradient, with the forward call's p, seed, t, worker and site; the
    residual's gradient is dy itself.  ``out`` may be dy."""
    return dropout(dy, p, seed, t, worker, site, out=out)


def _images(t, name: str) -> Tuple[int, int, int, int, int]:
    """(N, S, C, image pitch, pixel pitch) of an [N, ..., C] tensor."""
    if t.dim() < 2:
        raise ValueError("%s must be [N, ..., C]" % name)
    N, *pixels, C = t.shape
    S = math.prod(pixels)
    if C >> 31:
        _int(C, 32, "the number of channels")
    if t.is_contiguous():
        return N, S, C, S * C, C
    if t.stride(-1) != 1 and C > 1:
        raise ValueError("%s needs contiguous channels" % name)
    pixel, step = None, 0
    for k in range(t.dim() - 2, 0, -1):
        if t.shape[k] == 1:
            continue
        if pixel is None:
            pixel = step = t.stride(k)
        elif t.stride(k) != step:
            raise ValueError("%s needs evenly spaced pixels" % name)
        step *= t.shape[k]
    return N, S, C, t.stride(0), C if pixel is None else pixel


def _workspace(n: int, what: str, ref):
    if n < 0:
        raise GmcError(-1, load().gmc_last_error(None).decode() if what is None else what)
    return ref.new_empty(n, dtype=_torch().uint8) if n else None


def group_norm(x, groups: int, gamma=None, beta=None, eps: float = 1e-5, act: str = "none", out=None):
    """Group norm over channels-last x [N, ..., C] and its activation ("none",
    "relu", "silu"): (y, mean, rstd), the last two [N, groups] for the backward
    call.  gamma and beta are fp32 [C] (or None).  ``out`` may be x."""
    code = _code(x, "x")
    if act not in ACTS:
        raise ValueError("act must be one of %s" % list(ACTS))
    N, S, C, image, pixel = _images(x, "x")
    pg, pb = _f32(gamma, (C,), x, "gamma"), _f32(beta, (C,), x, "beta")
    if out is None:
        out = _new_like(x)
        oi, op = S * C, C
    else:
        _is(out, x.dtype, x.shape, x, "out")
        oi, op = _images(out, "out")[3:]
    G = int(groups)
    if G >> 31:
        _int(G, 32, "groups")
    lib = load()
    n = lib.gmc_group_norm_workspace(code, N, S, C, G, 0)
    ws = _workspace(n, None, x)
    mean = _new(x, N, G)
    rstd = _another(mean, x)
    _call(x, lib.gmc_group_norm, code, N, S, C, G, x.data_ptr(), image, pixel, pg, pb, float(eps), ACTS[act],
          out.data_ptr(), oi, op, mean.data_ptr(), rstd.data_ptr(), 0 if ws is None else ws.data_ptr(), n)
    return out, mean, rstd


def group_norm_backward(dy, x, mean, rstd, gamma=None, beta=None, act: str = "none", out=None, dgamma=None, dbeta=None):
    """(dx, dgamma, dbeta) from dy and the forward call's x, mean, rstd, gamma,
    beta and act.  ``out`` may be dy or x; ``dgamma`` and ``dbeta`` may be fp32
    [C] views of a worker's row of gradients."""
    code = _code(x, "x")
    _is(dy, x.dtype, x.shape, x, "dy")
    if act not in ACTS:
        raise ValueError("act must be one of %s" % list(ACTS))
    N, S, C, image, pixel = _images(x, "x")
    _, _, _, di, dp = _images(dy, "dy")
    if mean is None or rstd is None or mean.dim() != 2:
        raise ValueError("mean and rstd must be [N, groups]")
    G = int(mean.shape[1])
    if G >> 31:
        _int(G, 32, "groups")
    pm, ps = _f32(mean, (N, G), x, "mean"), _f32(rstd, (N, G), x, "rstd")
    pg, pb = _f32(gamma, (C,), x, "gamma"), _f32(beta, (C,), x, "beta")
    if out is None:
        out = _new_like(x)
        oi, op = S * C, C
    else:
        _is(out, x.dtype, x.shape, x, "out")
        oi, op = _images(out, "out")[3:]
    if dgamma is None:
        dgamma = _another(gamma, x, C)
    if dbeta is None:
        dbeta = _another(gamma, x, C)
    lib = load()
    n = lib.gmc_group_norm_workspace(code, N, S, C, G, 1)
    ws = _workspace(n, None, x)
    _call(x, lib.gmc_group_norm_backward, code, N, S, C, G, dy.data_ptr(), di, dp, x.data_ptr(), image, pixel, pm, ps,
          pg, pb, ACTS[act], out.data_ptr(), oi, op, _f32(dgamma, (C,), x, "dgamma"), _f32(dbeta, (C,), x, "dbeta"),
          0 if ws is None else ws.data_ptr(), n)
    return out, dgamma, dbeta


def _logits(logits, labels) -> Tuple[int, int, int, int, int, int]:
    """(code, R, T, V, label pointer, label pitch); without labels the last two are 0."""
    torch = _torch()
    code = _code(logits, "logits")
    if logits.dim() != 3:
        raise ValueError("logits must be [sequences, tokens, vocabulary]")
    R, T, V = logits.shape
    if V > 1 and logits.stride(2) != 1:
        raise ValueError("logits need a contiguous vocabulary axis")
    if labels is None:
        return code, R, T, V, 0, 0
    _is(labels, torch.int64, (R, T), logits, "labels")
    if T > 1 and labels.stride(1) != 1:
        raise ValueError("labels need contiguous tokens")
    return code, R, T, V, labels.data_ptr(), labels.stride(0)


def _labels(labels):
    if labels is None:
        raise TypeError("labels must be a torch.Tensor")
    return labels


def _gradient(logits, grad: bool, out):
    """(tensor or None, pointer, sequence pitch, token pitch) of the gradient.  A new
    one has the logits' strides where they are at most a quarter wider than dense: its
    rows then lie in lines as the logits' do, which the kernels read and write faster
    than rows that lie differently."""
    if out is not None:
        if not grad:
            raise ValueError("out is the gradient's: it needs grad=True")
        _is(out, logits.dtype, logits.shape, logits, "out")
        if out.shape[2] > 1 and out.stride(2) != 1:
            raise ValueError("out needs a contiguous vocabulary axis")
        return out, out.data_ptr(), out.stride(0), out.stride(1)
    R, T, V = logits.shape
    seq, tok = T * V, V
    if logits.is_contiguous():
        out = _torch().empty_like(logits) if grad else None
    else:
        s, k, _ = logits.stride()
        like = T > 1 and k >= V and s >= T * k and 4 * ((R - 1) * s + (T - 1) * k + V) <= 5 * R * T * V
        if like:
            seq, tok = s, k
        if grad:
            out = (_torch().empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=logits.device)
                   if like else logits.new_empty(logits.shape))
    return out, 0 if out is None else out.data_ptr(), seq, tok


def policy_loss(logits, labels, old_logp, advantages, ref_logp=None, clip: Tuple[float, float] = (0.2, 0.2),
                kl_coef: float = 0.0, temperature: float = 1.0, reduction: str = "token", ignore: int = IGNORE,
                grad: bool = True, grad_scale: float = 1.0, out=None):
    """The clipped policy loss of logits [R, T, V] at labels [R, T] (int64;
    ``ignore`` marks tokens that do not count): (stats, logp, gradient), stats =
    fp32 [3]: loss, mean KL, clipped share.

    old_logp, ref_logp: fp32 [R, T] or None; advantages: fp32 [R] or [R, T];
    reduction: "token" or "sequence".  The gradient (None without ``grad``) is
    grad_scale times the loss's, with strides like the logits' where those are
    nearly dense; ``out`` may be logits."""
    torch = _torch()
    code, R, T, V, pl, lp = _logits(logits, _labels(labels))
    if reduction not in REDUCTIONS:
        raise ValueError("reduction must be one of %s" % list(REDUCTIONS))
    po, pr = _f32(old_logp, (R, T), logits, "old_logp"), _f32(ref_logp, (R, T), logits, "ref_logp")
    if not isinstance(advantages, torch.Tensor):
        raise TypeError("advantages must be a torch.Tensor")
    per_token = advantages.dim() == 2
    pa = _f32(advantages, (R, T) if per_token else (R,), logits, "advantages")
    out, pg, gs, gt = _gradient(logits, grad, out)
    lib, ignore = load(), int(ignore)
    if ignore >> 63 not in (0, -1):
        _int(ignore, 64, "ignore")
    n = lib.gmc_policy_loss_workspace(R, T)
    ws = _workspace(n, "gmc_policy_loss: more than 2^22 - 1 tokens", logits)
    stats, logp = _new(logits, 3), _another(old_logp, logits, R, T)
    _call(logits, lib.gmc_policy_loss, code, R, T, V, logits.data_ptr(), logits.stride(0), logits.stride(1), pl, lp,
          ignore, po, pr, pa, T if per_token else 1, 1 if per_token else 0, float(clip[0]), float(clip[1]),
          float(kl_coef), float(temperature), REDUCTIONS[reduction], float(grad_scale), stats.data_ptr(),
          logp.data_ptr(), pg, gs, gt, ws.data_ptr(), n)
    return stats, logp, out


def preference_loss(logits, labels, ref_logp=None, beta: float = 0.1, smoothing: float = 0.0, average: bool = False,
                    ignore: int = IGNORE, grad: bool = True, grad_scale: float = 1.0, out=None):
    """The preference loss of P pairs, logits [2 P, T, V] with the chosen answers
    first: (loss, pair losses [P], rewards [2 P], logp [2 P, T], gradient).

    ref_logp: the reference's token log-probabilities, fp32 [2 P, T], as a call
    of its own with grad=False returns them, or None.  ``out`` may be logits."""
    code, R, T, V, pl, lp = _logits(logits, _labels(labels))
    if R % 2:
        raise ValueError("logits must hold pairs: [2 P, T, V]")
    P = R // 2
    pr = _f32(ref_logp, (R, T), logits, "ref_logp")
    out, pg, gs, gt = _gradient(logits, grad, out)
    lib, ignore = load(), int(ignore)
    if ignore >> 63 not in (0, -1):
        _int(ignore, 64, "ignore")
    n = lib.gmc_preference_loss_workspace(P, T)
    ws = _workspace(n, "gmc_preference_loss: more than 2^22 - 1 tokens", logits)
    loss, each, rewards, logp = _new(logits), _new(logits, P), _new(logits, R), _another(ref_logp, logits, R, T)
    _call(logits, lib.gmc_preference_loss, code, P, T, V, logits.data_ptr(), logits.stride(0), logits.stride(1), pl, lp,
          ignore, pr, float(beta), float(smoothing), 1 if average else 0, float(grad_scale), loss.data_ptr(),
          each.data_ptr(), rewards.data_ptr(), logp.data_ptr(), pg, gs, gt, 0 if ws is None else ws.data_ptr(), n)
    return loss, each, rewards, logp, out


def token_scores(logits, labels=None, top: int = 0, temperature: float = 1.0, ignore: int = IGNORE):
    """The scores of tokens with logits [R, T, V]: (logp, entropy, top_logp, top_ids,
    norm).

    logp: fp32 [R, T], the log-probabilities of ``labels`` (int64 [R, T], ``ignore``
    marks tokens that are not looked at; None: all are, and logp is None); entropy:
    fp32 [R, T]; top_logp, top_ids: fp32 and int64 [R, T, top], the ``top`` (up to 32)
    most probable tokens, equal ones by their place (None without ``top``); norm:
    fp32 [R, T, 2], the largest logit and the log of the sum, for the backward call."""
    torch = _torch()
    code, R, T, V, pl, lp = _logits(logits, labels)
    lib, ignore, top = load(), int(ignore), int(top)
    if ignore >> 63 not in (0, -1):
        _int(ignore, 64, "ignore")
    if top >> 31:
        _int(top, 32, "top")
    n = lib.gmc_token_scores_workspace(code, R, T, V, top)
    ws = _workspace(n, "gmc_token_scores: top must be in 0 to 32 and no more than the vocabulary, tokens below 2^22",
                    logits)
    # each result is a tensor of its own: views of one would share its version, so that an edit of one in place
    # is an edit of all to a backward pass that kept them
    norm, entropy = _new(logits, R, T, 2), _new(logits, R, T)
    logp = top_logp = top_ids = None
    if labels is not None:
        logp = torch.empty_like(entropy)
    if top:
        top_logp = _new(logits, R, T, top)
        top_ids = logits.new_empty((R, T, top), dtype=torch.int64)
    _call(logits, lib.gmc_token_scores, code, R, T, V, logits.data_ptr(), logits.stride(0), logits.stride(1), pl, lp,
          ignore, top, float(temperature), 0 if logp is None else logp.data_ptr(), entropy.data_ptr(),
          0 if top_logp is None else top_logp.data_ptr(), 0 if top_ids is None else top_ids.data_ptr(),
          norm.data_ptr(), 0 if ws is None else ws.data_ptr(), n)
    return logp, entropy, top_logp, top_ids, norm


def token_scores_backward(logits, norm, labels=None, dlogp=None, entropy=None, dentropy=None, top_ids=None, dtop=None,
                          temperature: float = 1.0, ignore: int = IGNORE, out=None):
    """The logits' gradient, with the forward call's logits, norm, labels, temperature
    and ignore, from the gradients of its results: dlogp and dentropy (fp32 [R, T]; the
    latter with the forward call's entropy) and dtop (fp32 [R, T, k], of the
    log-probabilities of top_ids, any k up to 32 tokens; one outside the vocabulary has
    no part).  The gradient has strides like the logits' where those are nearly dense;
    ``out`` may be logits."""
    torch = _torch()
    code, R, T, V, pl, lp = _logits(logits, labels)
    out, pg, gs, gt = _gradient(logits, True, out)
    pn = _f32(norm, (R, T, 2), logits, "norm")
    pd, ph = _f32(dlogp, (R, T), logits, "dlogp"), _f32(dentropy, (R, T), logits, "dentropy")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy needs entropy")
    if (top_ids is None) != (dtop is None):
        raise ValueError("top_ids and dtop come together")
    pe = _f32(entropy, (R, T), logits, "entropy")
    top = pi = 0
    if top_ids is not None:
        if top_ids.dim() != 3:
            raise ValueError("top_ids must be [R, T, k]")
        top = top_ids.shape[2]
        if top >> 31:
            _int(top, 32, "the number of top_ids")
        _is(top_ids, torch.int64, (R, T, top), logits, "top_ids")
        if not top_ids.is_contiguous():
            raise ValueError("top_ids must be contiguous")
        pi = top_ids.data_ptr()
    pt = _f32(dtop, (R, T, top), logits, "dtop")
    ignore = int(ignore)
    if ignore >> 63 not in (0, -1):
        _int(ignore, 64, "ignore")
    _call(logits, load().gmc_token_scores_backward, code, R, T, V, logits.data_ptr(), logits.stride(0),
          logits.stride(1), pl, lp, ignore, top, float(temperature), pn, pe, pd, ph, pi, pt, pg, gs, gt)
    return out
