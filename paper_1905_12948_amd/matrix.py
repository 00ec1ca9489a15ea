"""Orthogonalised matrices of a flat vector (include/gmc.h), on torch tensors: the
server's update with its matrices taken towards orthogonal ones, alone or as the
server's step with its momentum.

As elsewhere in the binding the calls only marshal arguments; they run on torch's
current stream of the tensors' device.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

from .gmc import GMC_OK, GmcError, _check, _torch, load
from .worker import _call, _code

# the five usual steps of the iteration: a, b, c of X <- a X + b (X X^T) X + c (X X^T)^2 X, the coefficients that were
# published with the optimizer Muon (K. Jordan and others, 2024)
QUINTIC = (3.4445, -4.7750, 2.0315)
STEPS = 5


def _whole(v, name: str) -> int:
    """v as an int; a whole number of any type."""
    try:
        n = int(v)
        if not isinstance(v, str) and n == v:
            return n
    except (OverflowError, ValueError):   # infinite or NaN
        pass
    raise ValueError("%s must be a whole number, got %s" % (name, v))


# plans closed or dropped while a stream was captured: freeing one waits for the device, which would
# end the capture
_dropped = []


def _free_dropped():
    if _dropped and not _torch().cuda.is_current_stream_capturing():
        while True:
            try:
                lib, plan = _dropped.pop()
            except IndexError:   # none left, or another thread took it
                return
            lib.gmc_matrices_destroy(plan)


class Matrices:
    """A plan: which matrices a vector of ``d`` components holds.

    ``table``: (offset, rows, cols) or (offset, rows, cols, pitch) of each, rows ``pitch``
    components apart (cols, if not given); no two share a component.  ``scales``: each
    one's factor (default 1).  The plan belongs to ``device`` and may be shared by streams;
    it has to live as long as graphs that were captured with it.  Closed or dropped
    while the thread's current stream is captured it is freed later, with the next plan that
    is made, closed or dropped; while another thread captures in the global mode it is
    neither."""

    def __init__(self, d: int, table: Sequence[Sequence[int]], scales: Optional[Sequence[float]] = None, device="cuda"):
        torch = _torch()
        self._lib, self._plan = load(), None
        d, rows = _whole(d, "d"), [tuple(_whole(v, "the table's entry") for v in entry) for entry in table]
        if any(len(entry) not in (3, 4) for entry in rows):
            raise ValueError("an entry of the table is (offset, rows, cols) or (offset, rows, cols, pitch)")
        if scales is not None and len(scales) != len(rows):
            raise ValueError("scales must hold one factor for each matrix")
        if any(not -1 << 63 <= v < 1 << 63 for entry in rows for v in entry) or not -1 << 63 <= d < 1 << 63:
            raise ValueError("d and the table must be 64-bit integers")
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device must be a GPU device")
        _free_dropped()
        n = len(rows)
        column = ctypes.c_int64 * n
        offset, r, c = (column(*[entry[k] for entry in rows]) for k in range(3))
        pitch = column(*[entry[3] if len(entry) == 4 else entry[2] for entry in rows])
        factor = None if scales is None else (ctypes.c_double * n)(*[float(v) for v in scales])
        plan = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            self.device = torch.device("cuda", torch.cuda.current_device())
            st = self._lib.gmc_matrices_init(ctypes.byref(plan), d, n, offset, r, c, pitch, factor)
        if st != GMC_OK:
            raise GmcError(st, self._lib.gmc_last_error(None).decode())
        self._plan, self.d, self.n = plan, d, n
        self.workspace = int(self._lib.gmc_matrices_workspace(plan))

    def close(self):
        if getattr(self, "_plan", None):
            _dropped.append((self._lib, self._plan))
            self._plan = None
        _free_dropped()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _vector(plan: Matrices, t, name: str) -> int:
    """Pointer of a contiguous fp32 vector of the plan's length and device."""
    p = _check(t, _torch().float32, plan.d, name)
    if t.get_device() != plan.device.index:
        raise ValueError("%s must be on %s" % (name, plan.device))
    return p


def _typed(plan: Matrices, t, name: str) -> Tuple[int, int]:
    """(element type, pointer) of a contiguous vector of the plan's length and device."""
    code = _code(t, name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.numel() < plan.d:
        raise ValueError("%s needs at least %d elements, has %d" % (name, plan.d, t.numel()))
    if t.get_device() != plan.device.index:
        raise ValueError("%s must be on %s" % (name, plan.device))
    return code, t.data_ptr()


def _several(v) -> bool:
    """Whether v holds several values; a tensor or array of no axes does not."""
    try:
        len(v)
    except TypeError:
        return False
    return True


def _steps(steps: int, coefficients):
    """(number, host array) of the steps' coefficients: one triple for all, or one a step;
    sequences, arrays or tensors."""
    steps = _whole(steps, "steps")
    if not 1 <= steps <= 64:
        raise ValueError("steps must be in 1 to 64")
    values = None
    if _several(coefficients):
        if len(coefficients) == 3 and not _several(coefficients[0]):
            values = [float(v) for v in coefficients] * steps
        elif len(coefficients) == steps and all(_several(c) and len(c) == 3 and not _several(c[0]) for c in coefficients):
            values = [float(v) for c in coefficients for v in c]
    if values is None:
        raise ValueError("coefficients must be (a, b, c), or one such a step")
    return steps, (ctypes.c_double * (3 * steps))(*values)


def _plan_of(plan) -> Matrices:
    if not isinstance(plan, Matrices):
        raise TypeError("plan must be a Matrices")
    if not plan._plan:
        raise ValueError("the plan is closed")
    return plan


def orthogonalize(plan: Matrices, x, out=None, steps: int = STEPS, coefficients=QUINTIC, eps: float = 1e-7,
                  alpha: float = 1.0):
    """x (flat, fp32, bf16 or fp16) with every matrix M of the plan replaced by alpha *
    scale * X, X what ``steps`` steps X <- a X + b (X X^T) X + c (X X^T)^2 X make of
    M / (|M| + eps); the other components as they are.  ``coefficients``: (a, b, c), or
    one such a step.  ``out`` may be x; a new one has the plan's number of components where x
    has more."""
    plan = _plan_of(plan)
    torch = _torch()
    code, px = _typed(plan, x, "x")
    steps, c = _steps(steps, coefficients)
    if out is None:
        out = torch.empty_like(x) if x.numel() == plan.d else x.new_empty(plan.d)
        po = out.data_ptr()
    else:
        co, po = _typed(plan, out, "out")
        if co != code:
            raise TypeError("out must be %s, got %s" % (x.dtype, out.dtype))
    ws = x.new_empty(plan.workspace, dtype=torch.uint8)
    _call(x, plan._lib.gmc_orthogonalize, plan._plan, code, px, po, steps, c, float(eps), float(alpha), ws.data_ptr(),
          plan.workspace)
    return out


def orthogonal_step(plan: Matrices, w, update, momentum, rate: float, mu: float = 0.95, nesterov: bool = True,
                    decay: float = 0.0, w_out=None, steps: int = STEPS, coefficients=QUINTIC, eps: float = 1e-7):
    """The server's step from the update that Gmc.aggregate gives (a gradient takes a
    negative rate): in the matrices momentum = mu * momentum + update and w_out = (1 -
    decay) w + rate * scale * X, X from update + mu * momentum (``nesterov``) or
    momentum as in ``orthogonalize``; elsewhere w_out = w + update, as Gmc.apply.

    w, momentum, w_out: fp32; ``momentum`` is updated in place (None: none);
    ``w_out`` None: w is.  Returns w_out."""
    plan = _plan_of(plan)
    torch = _torch()
    pw = _vector(plan, w, "w")
    code, pu = _typed(plan, update, "update")
    pm = 0 if momentum is None else _vector(plan, momentum, "momentum")
    if w_out is None:
        w_out = w
    po = _vector(plan, w_out, "w_out")
    steps, c = _steps(steps, coefficients)
    ws = w.new_empty(plan.workspace, dtype=torch.uint8)
    _call(w, plan._lib.gmc_orthogonal_step, plan._plan, code, pw, pu, pm, po, float(rate), float(mu),
          1 if nesterov else 0, float(decay), steps, c, float(eps), ws.data_ptr(), plan.workspace)
    return w_out
