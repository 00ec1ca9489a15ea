"""Arguments the calls for tokens' scores and for plans of matrices refuse, before any
device work (no GPU: the pointers are never dereferenced), and workspace sizes."""
import ctypes
import os

import pytest

F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_1905_12948_amd import gmc
    if not os.path.exists(gmc.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return gmc.load()


def at(k):
    return (k + 1) << 32


NAMES = ("x", "labels", "logp", "entropy", "top_logp", "top_ids", "norm", "ws", "grad", "dlogp", "dentropy", "dtop")
PLACE = {n: at(k) for k, n in enumerate(NAMES)}
R, T, V, K = 3, 4, 60000, 5
CALL = dict(PLACE, dtype=F32, R=R, T=T, V=V, seq=T * V, tok=V, lp=T, ignore=-100, top=K, tau=1.0, n=1 << 30, gs=T * V, gt=V)


def forward(lib, **change):
    a = dict(CALL, **change)
    return lib.gmc_token_scores(None, a["dtype"], a["R"], a["T"], a["V"], a["x"], a["seq"], a["tok"], a["labels"], a["lp"],
                                a["ignore"], a["top"], a["tau"], a["logp"], a["entropy"], a["top_logp"], a["top_ids"],
                                a["norm"], a["ws"], a["n"])


def backward(lib, **change):
    a = dict(CALL, **change)
    return lib.gmc_token_scores_backward(None, a["dtype"], a["R"], a["T"], a["V"], a["x"], a["seq"], a["tok"], a["labels"],
                                         a["lp"], a["ignore"], a["top"], a["tau"], a["norm"], a["entropy"], a["dlogp"],
                                         a["dentropy"], a["top_ids"], a["dtop"], a["grad"], a["gs"], a["gt"])


def refused(lib, st, needle):
    said = lib.gmc_last_error(None).decode()
    assert st == -1 and needle in said, (st, said)


BOTH = [
    (dict(dtype=3), "type"), (dict(dtype=-1), "type"), (dict(R=-1), "R >= 0"), (dict(T=-1), "R >= 0"), (dict(V=0), "R >= 0"),
    (dict(V=1 << 30), "R >= 0"), (dict(R=1 << 20), "2^22"), (dict(x=None), "NULL"), (dict(tok=V - 1), "pitch"),
    (dict(seq=V), "pitch"), (dict(lp=T - 1), "label pitch"), (dict(top=-1), "top must"), (dict(top=33), "top must"),
    (dict(tau=0.0), "temperature"), (dict(tau=-1.0), "temperature"), (dict(tau=float("nan")), "temperature"),
    (dict(tau=1e-40), "temperature"), (dict(norm=None), "NULL"), (dict(norm=PLACE["norm"] + 4), "norm is not"),
    (dict(top_ids=None), "NULL"),
]


@pytest.mark.parametrize("change,needle", BOTH + [
    (dict(V=4, tok=4, seq=16), "top must"), (dict(entropy=None), "NULL"), (dict(logp=None), "NULL"), (dict(top_logp=None), "NULL"),
    (dict(R=1 << 21, T=1, V=1 << 29, tok=1 << 29, seq=1 << 29), "than a launch has"),
    (dict(ws=None), "workspace"), (dict(n=100), "workspace"), (dict(ws=PLACE["ws"] + 8), "aligned"),
])
def test_forward(lib, change, needle):
    refused(lib, forward(lib, **change), needle)


@pytest.mark.parametrize("change,needle", BOTH + [
    (dict(gt=V - 1), "pitch"), (dict(gs=V), "pitch"), (dict(grad=None), "NULL"), (dict(entropy=None), "NULL"),
    (dict(dtop=None), "NULL"), (dict(labels=None), "dlogp needs labels"),
    (dict(grad=PLACE["x"] + 4), "overlaps the logits"), (dict(grad=PLACE["x"], gt=V + 1, gs=T * V + T), "overlaps the logits"),
])
def test_backward(lib, change, needle):
    refused(lib, backward(lib, **change), needle)


BYTES = {"logp": R * T * 4, "entropy": R * T * 4, "top_logp": R * T * K * 4, "top_ids": R * T * K * 8, "norm": R * T * 8}


@pytest.mark.parametrize("a", list(BYTES))
@pytest.mark.parametrize("b", ["x", "labels", "ws", "logp", "norm"])
def test_forward_overlaps(lib, a, b):
    if a == b:
        return
    for shift in (0, BYTES[a] - 4):
        where = PLACE[a] + shift
        if b in ("ws", "norm"):
            where = where // 16 * 16
        refused(lib, forward(lib, **{b: where}), "overlaps another buffer")


@pytest.mark.parametrize("b", ["labels", "norm", "entropy", "dlogp", "dentropy", "top_ids", "dtop"])
def test_backward_overlaps(lib, b):
    for shift in (0, R * T * V * 4 - 8):
        refused(lib, backward(lib, **{b: PLACE["grad"] + shift}), "overlaps")


def test_nothing_to_do_needs_no_device(lib):
    assert forward(lib, R=0) == 0 and forward(lib, T=0) == 0
    assert backward(lib, R=0) == 0 and backward(lib, T=0) == 0


def test_workspaces(lib):
    size = lib.gmc_token_scores_workspace
    assert size(BF16, 4, 4, 1000, 5) == 0
    assert size(F32, 0, 4, 200000, 5) == 0 and size(F32, 1 << 40, 0, 200000, 5) == 0
    assert size(F32, 100, 10, 1000000, 8) > 1000 * 16
    for bad in ((3, 4, 4, 100, 5), (F32, -1, 4, 100, 5), (F32, 4, -1, 100, 5), (F32, 4, 4, 0, 0), (F32, 4, 4, 1 << 30, 0),
                (F32, 4, 4, 100, 33), (F32, 1 << 21, 1, 1 << 29, 0), (F32, 4, 4, 100, -1), (F32, 4, 4, 4, 5), (F32, 1 << 20, 1 << 20, 100, 5)):
        assert size(*bad) == -1, bad


# -- plans of matrices --------------------------------------------------------------


def plan(lib, d, table, scales=None, n=None, null=()):
    out = ctypes.c_void_p(77)
    k = len(table)
    column = ctypes.c_int64 * max(k, 1)
    cols = [column(*[e[i] for e in table]) for i in range(3)]
    pitch = column(*[e[3] if len(e) > 3 else e[2] for e in table])
    factor = None if scales is None else (ctypes.c_double * k)(*scales)
    given = [None if i in null else c for i, c in enumerate(cols)]
    st = lib.gmc_matrices_init(ctypes.byref(out), d, k if n is None else n, *given, pitch, factor)
    if st:
        assert not out.value      # a failed call leaves no plan
    return st


@pytest.mark.parametrize("d,table,needle", [
    (0, [], "1 <= d"), (-1, [], "1 <= d"), ((1 << 40) + 1, [], "1 <= d"),
    (10, [(0, 0, 5)], "rows and columns"), (10, [(0, 5, 0)], "rows and columns"), (10, [(0, -1, 5)], "rows and columns"),
    (1 << 40, [(0, 1, (1 << 26) + 1)], "rows and columns"), (100, [(0, 3, 5, 4)], "pitch"), (100, [(0, 3, 5, 101)], "pitch"),
    (10, [(-1, 2, 2)], "inside"), (10, [(10, 1, 1)], "inside"), (10, [(7, 2, 2)], "inside"), (10, [(0, 3, 4)], "inside"),
    (100, [(0, 1 << 26, 50)], "inside"), (1 << 40, [(0, 1 << 26, 1 << 26)], "inside"),
    (20, [(0, 2, 4), (7, 2, 2)], "share"), (20, [(7, 2, 2), (0, 2, 4)], "share"), (20, [(3, 2, 2), (3, 2, 2)], "share"),
    (40, [(0, 4, 5, 10), (4, 4, 5, 10)], "share"),        # columns that meet
    (40, [(2, 3, 5, 10), (7, 3, 6, 10)], "share"),        # columns that reach the next row's
    (40, [(0, 4, 5, 10), (5, 4, 4, 9)], "share"),         # other pitches
    (40, [(0, 4, 5, 10), (24, 1, 3)], "share"),           # one row over another's columns
    (40, [(0, 1, 20), (5, 2, 3, 10)], "share"),
    (1 << 40, [(0, 1 << 20, 1 << 20)], "tiles"),
    (1 << 40, [(0, 1 << 13, 1 << 13), (1 << 26, 1 << 20, 1 << 19)], "tiles"),
    (1 << 40, [(0, 1 << 26, 1, 2), (1, 1 << 26, 1, 2)], "rows that are apart"),
])
def test_plan_refusals(lib, d, table, needle):
    refused(lib, plan(lib, d, table), needle)


def test_plan_counts_and_scales(lib):
    refused(lib, plan(lib, 10, [], n=-1), "8192")
    refused(lib, plan(lib, 10, [(0, 2, 2)], n=8193), "8192")
    refused(lib, plan(lib, 10, [(0, 2, 2)], null=(0,)), "NULL")
    refused(lib, plan(lib, 10, [(0, 2, 2)], null=(2,)), "NULL")
    for bad in (float("nan"), float("inf"), 1e39):
        refused(lib, plan(lib, 10, [(0, 2, 2)], scales=[bad]), "scale")
    assert lib.gmc_matrices_init(None, 10, 0, None, None, None, None, None) == -1


def test_calls_without_a_plan(lib):
    coef = (ctypes.c_double * 3)(1.5, -0.5, 0.0)
    refused(lib, lib.gmc_orthogonalize(None, None, F32, 1 << 20, 1 << 30, 1, coef, 1e-7, 1.0, 1 << 40, 1 << 20), "NULL")
    refused(lib, lib.gmc_orthogonal_step(None, None, F32, 1 << 20, 1 << 30, None, 1 << 40, 0.1, 0.9, 1, 0.0, 1, coef, 1e-7,
                                         1 << 50, 1 << 20), "NULL")
    assert lib.gmc_matrices_workspace(None) == -1
    lib.gmc_matrices_destroy(None)
