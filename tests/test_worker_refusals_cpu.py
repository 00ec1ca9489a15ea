"""Arguments the worker-side operators refuse, before any device work (no GPU:
the pointers are never dereferenced), and their workspace sizes."""
import ctypes
import os

import pytest

P = ctypes.c_void_p(1 << 20)
Q = ctypes.c_void_p(1 << 40)
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_1905_12948_amd import gmc
    if not os.path.exists(gmc.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return gmc.load()


def refused(lib, st, needle):
    assert st == -1
    assert needle in lib.gmc_last_error(None).decode(), lib.gmc_last_error(None)


DROP = dict(dtype=BF16, rows=4, cols=8, x=P, xp=8, r=None, rp=0, y=Q, yp=8, p=0.1, seed=1, t=0, worker=0, site=0)


@pytest.mark.parametrize("change,needle", [
    (dict(dtype=3), "type"), (dict(dtype=-1), "type"), (dict(rows=-1), "rows"), (dict(cols=-1), "rows"),
    (dict(p=-0.1), "p must"), (dict(p=1.1), "p must"), (dict(p=float("nan")), "p must"), (dict(t=-1), "need t"),
    (dict(worker=-1), "need t"), (dict(worker=64), "need t"), (dict(site=-1), "need t"), (dict(x=None), "NULL"),
    (dict(y=None), "NULL"), (dict(xp=7), "pitch"), (dict(yp=0), "pitch"), (dict(r=P, rp=7), "pitch"),
    (dict(rows=1 << 30, cols=1 << 12, xp=1 << 12, yp=1 << 12), "2^40"), (dict(xp=1 << 60), "2^40"),
    (dict(y=ctypes.c_void_p((1 << 20) + 2)), "overlaps"), (dict(y=P, yp=9), "overlaps"),
])
def test_dropout(lib, change, needle):
    a = dict(DROP, **change)
    refused(lib, lib.gmc_dropout(None, a["dtype"], a["rows"], a["cols"], a["x"], a["xp"], a["r"], a["rp"], a["y"], a["yp"],
                                 a["p"], a["seed"], a["t"], a["worker"], a["site"]), needle)


def test_nothing_to_do_needs_no_device(lib):
    assert lib.gmc_dropout(None, F32, 0, 8, None, 0, None, 0, None, 0, 0.1, 1, 0, 0, 0) == 0
    assert lib.gmc_dropout(None, F32, 8, 0, None, 0, None, 0, None, 0, 0.1, 1, 0, 0, 0) == 0
    assert lib.gmc_group_norm(None, F32, 0, 4, 8, 2, None, 0, 0, None, None, 1e-5, 0, None, 0, 0, None, None, None, 0) == 0
    assert lib.gmc_group_norm_workspace(F32, 0, 4, 8, 2, 1) == 0


NORM = dict(dtype=BF16, N=2, S=6, C=8, G=2, x=P, xi=48, xp=8, eps=1e-5, act=0, y=Q, yi=48, yp=8, mean=P, rstd=P, ws=P,
            n=1 << 20)


@pytest.mark.parametrize("change,needle", [
    (dict(dtype=9), "type"), (dict(N=-1), "N >= 0"), (dict(S=0), "N >= 0"), (dict(S=1 << 31), "N >= 0"),
    (dict(C=0), "N >= 0"), (dict(G=0), "multiple"), (dict(G=3), "multiple"), (dict(act=3), "activation"),
    (dict(act=-1), "activation"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(x=None), "NULL"),
    (dict(y=None), "NULL"), (dict(mean=None), "NULL"), (dict(rstd=None), "NULL"), (dict(xp=7), "pitch"),
    (dict(yi=47), "pitch"), (dict(N=1 << 40), "2^40"), (dict(y=ctypes.c_void_p((1 << 20) + 16)), "overlaps"),
])
def test_group_norm(lib, change, needle):
    a = dict(NORM, **change)
    refused(lib, lib.gmc_group_norm(None, a["dtype"], a["N"], a["S"], a["C"], a["G"], a["x"], a["xi"], a["xp"], None, None,
                                    a["eps"], a["act"], a["y"], a["yi"], a["yp"], a["mean"], a["rstd"], a["ws"], a["n"]),
            needle)
    if "eps" in change or "mean" in change or "rstd" in change:
        return
    R = ctypes.c_void_p(1 << 50)
    refused(lib, lib.gmc_group_norm_backward(None, a["dtype"], a["N"], a["S"], a["C"], a["G"], R, 48, 8, a["x"], a["xi"],
                                             a["xp"], P, P, None, None, a["act"], a["y"], a["yi"], a["yp"], P, P, a["ws"],
                                             a["n"]), needle)


def test_group_norm_workspace(lib):
    assert lib.gmc_group_norm_workspace(BF16, 2, 6, 8, 3, 0) == -1
    assert lib.gmc_group_norm_workspace(BF16, 2, 0, 8, 2, 0) == -1
    need = lib.gmc_group_norm_workspace(BF16, 2, 6, 8, 2, 1)
    assert need > 0
    refused(lib, lib.gmc_group_norm_backward(None, BF16, 2, 6, 8, 2, P, 48, 8, P, 48, 8, P, P, None, None, 0, Q, 48, 8, P, P,
                                             P, need - 1), "workspace")
    refused(lib, lib.gmc_group_norm_backward(None, BF16, 2, 6, 8, 2, P, 48, 8, P, 48, 8, P, P, None, None, 0, Q, 48, 8, P, P,
                                             None, need), "workspace")


LOSS = dict(dtype=BF16, R=4, T=3, V=10, x=P, xs=30, xt=10, labels=P, lp=3, old=None, ref=None, adv=P, lo=0.2, hi=0.2,
            kl=0.0, tau=1.0, scale=1.0, stats=P, logp=P, g=Q, gs=30, gt=10, ws=P, n=1 << 20)
BOTH = [
    (dict(dtype=5), "type"), (dict(T=-1), "need R"), (dict(V=0), "need R"), (dict(V=1 << 30), "need R"),
    (dict(x=None), "NULL"), (dict(labels=None), "NULL"), (dict(logp=None), "NULL"), (dict(xt=9), "pitch"),
    (dict(xs=29), "pitch"), (dict(gt=9), "pitch"), (dict(gs=29), "pitch"), (dict(lp=2), "label pitch"),
    (dict(T=1 << 22), "2^22"), (dict(ws=None), "workspace"), (dict(n=8), "workspace"),
    (dict(ws=ctypes.c_void_p((1 << 20) + 4)), "aligned"), (dict(stats=None), "NULL"),
    (dict(g=ctypes.c_void_p((1 << 20) + 20)), "overlaps"), (dict(g=P, gt=11, gs=33), "overlaps"),
    (dict(scale=float("inf")), "finite"),
]


@pytest.mark.parametrize("change,needle", BOTH + [
    (dict(R=-1), "need R"), (dict(adv=None), "NULL"), (dict(lo=-0.1), "clip"), (dict(lo=1.1), "clip"), (dict(hi=-0.1), "clip"),
    (dict(hi=float("nan")), "clip"), (dict(kl=float("nan")), "finite"), (dict(tau=0.0), "temperature"),
    (dict(tau=float("inf")), "temperature"),
])
def test_policy_loss(lib, change, needle):
    a = dict(LOSS, **change)
    refused(lib, lib.gmc_policy_loss(None, a["dtype"], a["R"], a["T"], a["V"], a["x"], a["xs"], a["xt"], a["labels"], a["lp"],
                                     -100, a["old"], a["ref"], a["adv"], 1, 0, a["lo"], a["hi"], a["kl"], a["tau"], 0,
                                     a["scale"], a["stats"], a["logp"], a["g"], a["gs"], a["gt"], a["ws"], a["n"]), needle)


@pytest.mark.parametrize("change,needle", BOTH + [
    (dict(R=-2), "P"), (dict(kl=float("inf")), "finite"), (dict(lo=-0.1), "smoothing"), (dict(lo=1.5), "smoothing"),
])
def test_preference_loss(lib, change, needle):
    a = dict(LOSS, **change)  # kl is beta here, lo the smoothing
    refused(lib, lib.gmc_preference_loss(None, a["dtype"], a["R"] // 2, a["T"], a["V"], a["x"], a["xs"], a["xt"], a["labels"],
                                         a["lp"], -100, None, a["kl"], a["lo"], 0, a["scale"], a["stats"], P, P, a["logp"],
                                         a["g"], a["gs"], a["gt"], a["ws"], a["n"]), needle)


def test_loss_workspaces(lib):
    assert lib.gmc_policy_loss_workspace(-1, 3) == -1 and lib.gmc_policy_loss_workspace(1 << 12, 1 << 12) == -1
    assert lib.gmc_preference_loss_workspace(1, -1) == -1 and lib.gmc_preference_loss_workspace(1 << 12, 1 << 12) == -1
    assert lib.gmc_policy_loss_workspace(4, 8) > 0 and lib.gmc_preference_loss_workspace(4, 8) > 0


def test_binding_refuses_before_device_work():
    torch = pytest.importorskip("torch")
    import paper_1905_12948_amd as gmc
    cpu = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError):
        gmc.dropout(cpu, 0.1, 1)                       # not on a GPU
    with pytest.raises(TypeError):
        gmc.dropout(cpu.double(), 0.1, 1)
    with pytest.raises(TypeError):
        gmc.group_norm(cpu.long(), 2)
    with pytest.raises(ValueError):
        gmc.policy_loss(cpu, torch.zeros(2, 3, dtype=torch.int64), None, torch.zeros(2))
    with pytest.raises(TypeError):
        gmc.preference_loss([1.0], None)
