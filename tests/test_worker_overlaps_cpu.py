"""Buffers the worker-side operators refuse to share: an output or the workspace over
an input, another output or the workspace (no GPU: the pointers are never dereferenced)."""
import ctypes
import os

import pytest

BF16 = 1


@pytest.fixture(scope="module")
def lib():
    from paper_1905_12948_amd import gmc
    if not os.path.exists(gmc.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return gmc.load()


def apart(names):
    """Pointers a gigabyte apart."""
    return {n: (k + 1) << 30 for k, n in enumerate(names)}


def shared(lib, call, places, a, b, bytes_of_a):
    """`call` refuses b where it begins at a or in its last bytes."""
    for shift in (0, bytes_of_a - 2):
        p = dict(places)
        p[b] = p[a] + shift
        st = call({k: ctypes.c_void_p(v) for k, v in p.items()})
        said = lib.gmc_last_error(None).decode()
        assert st == -1 and "overlaps another buffer" in said, (a, b, shift, st, said)


N, S, C, G = 2, 6, 8, 2
IMAGE = ("x", "dy", "out", "gamma", "beta", "mean", "rstd", "dgamma", "dbeta", "ws")
SIZE = {"mean": 4 * N * G, "rstd": 4 * N * G, "dgamma": 4 * C, "dbeta": 4 * C, "out": 2 * N * S * C}


@pytest.mark.parametrize("a,b", [("mean", "rstd"), ("mean", "x"), ("rstd", "x"), ("mean", "gamma"), ("rstd", "beta"),
                                 ("mean", "out"), ("rstd", "out"), ("out", "gamma"), ("out", "beta")])
def test_group_norm(lib, a, b):
    def call(p):
        return lib.gmc_group_norm(None, BF16, N, S, C, G, p["x"], S * C, C, p["gamma"], p["beta"], 1e-5, 0, p["out"], S * C, C,
                                  p["mean"], p["rstd"], p["ws"], 0)
    shared(lib, call, apart(IMAGE), a, b, SIZE[a])


@pytest.mark.parametrize("a,b", [("dgamma", "dbeta"), ("dgamma", "gamma"), ("dgamma", "beta"), ("dbeta", "gamma"),
                                 ("dbeta", "beta"), ("dgamma", "x"), ("dbeta", "dy"), ("dgamma", "mean"), ("dbeta", "rstd"),
                                 ("dgamma", "out"), ("out", "gamma"), ("out", "mean"), ("out", "rstd"), ("dgamma", "ws"),
                                 ("out", "ws")])
def test_group_norm_backward(lib, a, b):
    need = lib.gmc_group_norm_workspace(BF16, N, S, C, G, 1)

    def call(p):
        return lib.gmc_group_norm_backward(None, BF16, N, S, C, G, p["dy"], S * C, C, p["x"], S * C, C, p["mean"], p["rstd"],
                                           p["gamma"], p["beta"], 0, p["out"], S * C, C, p["dgamma"], p["dbeta"], p["ws"], need)
    shared(lib, call, apart(IMAGE), a, b, SIZE[a])


R, T, V = 4, 3, 10
TOKENS = ("logits", "labels", "old", "ref", "adv", "stats", "logp", "grad", "ws", "each", "rewards")
LOSS_SIZE = {"logp": 4 * R * T, "stats": 12, "grad": 2 * R * T * V, "loss": 4, "each": 2 * R, "rewards": 4 * R}


@pytest.mark.parametrize("a,b", [("logp", "old"), ("logp", "ref"), ("logp", "labels"), ("logp", "adv"), ("logp", "logits"),
                                 ("logp", "stats"), ("logp", "grad"), ("stats", "adv"), ("stats", "logits"), ("grad", "labels"),
                                 ("grad", "old"), ("grad", "adv"), ("logp", "ws"), ("stats", "ws"), ("grad", "ws")])
def test_policy_loss(lib, a, b):
    n = lib.gmc_policy_loss_workspace(R, T)

    def call(p):
        shift = p["ws"].value % 16  # the workspace's own alignment is not what is refused here
        ws = ctypes.c_void_p(p["ws"].value - shift)
        return lib.gmc_policy_loss(None, BF16, R, T, V, p["logits"], T * V, V, p["labels"], T, -100, p["old"], p["ref"], p["adv"],
                                   1, 0, 0.2, 0.2, 0.1, 1.0, 0, 1.0, p["stats"], p["logp"], p["grad"], T * V, V, ws, n)
    shared(lib, call, apart(TOKENS), a, b, LOSS_SIZE[a])


@pytest.mark.parametrize("a,b", [("logp", "ref"), ("logp", "labels"), ("logp", "logits"), ("logp", "rewards"), ("logp", "each"),
                                 ("logp", "stats"), ("logp", "grad"), ("rewards", "each"), ("rewards", "ref"), ("each", "stats"),
                                 ("grad", "labels"), ("grad", "ref"), ("grad", "ws"), ("logp", "ws"), ("rewards", "ws")])
def test_preference_loss(lib, a, b):
    n = lib.gmc_preference_loss_workspace(R // 2, T)

    def call(p):
        ws = ctypes.c_void_p(p["ws"].value - p["ws"].value % 8)
        return lib.gmc_preference_loss(None, BF16, R // 2, T, V, p["logits"], T * V, V, p["labels"], T, -100, p["ref"], 0.1, 0.0, 0,
                                       1.0, p["stats"], p["each"], p["rewards"], p["logp"], p["grad"], T * V, V, ws, n)
    shared(lib, call, apart(TOKENS), a, b, LOSS_SIZE[a])


def test_advantages_read_backwards(lib):
    """Negative pitches: the range that is read lies below the pointer."""
    n = lib.gmc_policy_loss_workspace(R, T)
    p = apart(TOKENS)
    p["logp"] = p["adv"] - 8
    p = {k: ctypes.c_void_p(v) for k, v in p.items()}
    st = lib.gmc_policy_loss(None, BF16, R, T, V, p["logits"], T * V, V, p["labels"], T, -100, p["old"], p["ref"], p["adv"], -1, 0,
                             0.2, 0.2, 0.1, 1.0, 0, 1.0, p["stats"], p["logp"], p["grad"], T * V, V, p["ws"], n)
    assert st == -1 and "overlaps another buffer" in lib.gmc_last_error(None).decode()
    st = lib.gmc_policy_loss(None, BF16, R, T, V, p["logits"], T * V, V, p["labels"], T, -100, p["old"], p["ref"], p["adv"],
                             1 << 60, 0, 0.2, 0.2, 0.1, 1.0, 0, 1.0, p["stats"], p["logp"], p["grad"], T * V, V, p["ws"], n)
    assert st == -1 and "advantages" in lib.gmc_last_error(None).decode()
