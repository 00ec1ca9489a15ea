"""How group norm's plan (csrc/gmc_norm_plan.h) lays a call out: compiled for the host
and asked by shape, so that a list of shapes can be held against the kernels it reaches."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FIELDS = ("held", "fold", "vec", "threads", "kp", "lds", "gw", "cb", "blocks", "tc", "tp_log2", "once", "chunk", "chunks",
          "cblocks", "images")
SOURCE = r'''
#include "%s"
extern "C" void plan(int64_t size, int64_t N, int32_t S, int32_t C, int32_t G, int32_t backward, int64_t* out) {
    gmc::NormArgs a{};
    a.N = N, a.S = S, a.C = C, a.G = G, a.out_pixel = C;
    const gmc::NormPlan p = gmc::norm_plan(a, size, backward != 0);
    const int64_t v[] = {p.held, p.fold, p.vec, p.threads, p.kp, (int64_t)p.lds, a.gw, a.cb, a.blocks, a.tc, a.tp_log2, a.once,
                         a.chunk, a.chunks, a.cblocks, gmc::launch_images(a, p, backward != 0)};
    for (int i = 0; i < 16; ++i) out[i] = v[i];
}
'''


def build(folder):
    """plan(size, N, S, C, G, backward) -> dict of the plan's fields."""
    source, lib = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan.so")
    with open(source, "w") as f:
        f.write(SOURCE % os.path.join(ROOT, "paper_1905_12948_amd", "csrc", "gmc_norm_plan.h"))
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", source, "-o", lib], check=True)
    f = ctypes.CDLL(lib).plan
    f.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]

    def plan(size, N, S, C, G, backward):
        out = (ctypes.c_int64 * 16)()
        f(size, N, S, C, G, backward, out)
        return dict(zip(FIELDS, out))
    return plan


def kernel(p, size, backward):
    """The kernel a plan runs: (form, bytes of an element, vectors a thread or None, groups in a
    vector or channels of a thread), as the entry points choose it."""
    if p["fold"]:
        held = ((2, 4, 8) if backward else (4, 8, 16))
        return "fold", size, next(h for h in held if p["kp"] <= h), p["fold"]
    if p["held"]:
        return "held", size, p["kp"], p["vec"]
    return "split", size, None, p["vec"]


def kernels(backward):
    """Every kernel there is."""
    fold = [("fold", size, kp, F) for size in (2, 4) for kp in ((2, 4, 8) if backward else (4, 8, 16))
            for F in ((1, 2, 4, 8) if size == 2 else (1, 2, 4))]
    held = [("held", size, kp, vec) for size in (2, 4) for kp in ((4, 8) if backward else (4, 16)) for vec in (1, 16 // size)]
    return set(fold + held + [("split", size, None, vec) for size in (2, 4) for vec in (1, 16 // size)])


def branches(p, size, N, S, C, G, backward):
    """The choices of the plan, beside the kernel, that a call's layout went through."""
    out = set()
    if p["fold"]:
        wide = p["cb"] * size
        out.add(("line", 128 if wide >= 128 else 64 if wide >= 64 else 32 if wide >= 32 else 16))
        out.add(("workgroups", "512" if N * p["blocks"] >= 512 else "256" if N * p["blocks"] >= 256 else "few"))
        out.add(("threads", p["threads"]))
        out.add(("whole lines", p["once"]))
        out.add(("lanes that idle", p["tc"] != 1 << p["tp_log2"]))
        out.add(("pixels fill the threads", S % (p["threads"] >> p["tp_log2"]) == 0))
        if p["lds"] > 65536:
            out.add(("LDS above 64 KB",))
    elif p["held"]:
        out.add(("held threads", p["threads"]))
        out.add(("held across wavefronts", p["tp_log2"] >= 6))
        out.add(("held blocks", p["blocks"] > 1))
    else:
        cpg = C // G
        out.add(("split of narrow blocks", backward and cpg & (cpg - 1) == 0 and cpg <= 64 and N * S * C * size >= 48 << 20))
        out.add(("split blocks", p["cblocks"] > 1))
        out.add(("split chunks", "one" if p["chunks"] == 1 else "even" if S % p["chunk"] == 0 else "ragged"))
        out.add(("split across wavefronts", p["tp_log2"] >= 6))
        out.add(("split lanes that idle", p["tc"] != 1 << p["tp_log2"]))
    return out


SHAPES = [  # N, S, C, G; test_worker_forms_cpu.py holds them against every kernel and branch, in 16 and 32 bits
    # groups of a power of two of channels, few images: all widths of a block, lane and vector counts
    (3, 5, 8, 1), (2, 7, 8, 2), (2, 6, 8, 4), (3, 9, 8, 8), (2, 5, 4, 1), (2, 5, 4, 2), (2, 5, 4, 4), (5, 3, 24, 3), (2, 16, 32, 1),
    (1, 65, 32, 1), (1, 129, 8, 1), (1, 132, 8, 2), (1, 140, 8, 4), (1, 136, 8, 8), (1, 130, 32, 1), (1, 33, 16, 1), (1, 156, 4, 2),
    (1, 129, 4, 4), (1, 1040, 8, 8), (1, 513, 64, 1), (1, 2051, 16, 1), (1, 2089, 32, 1), (1, 4141, 8, 2), (1, 4433, 8, 2),
    (1, 4139, 8, 4), (1, 4549, 8, 8), (1, 8367, 8, 2), (1, 8578, 8, 4), (1, 8372, 8, 8), (1, 1057, 16, 1), (1, 4171, 4, 2),
    (1, 4423, 4, 4), (1, 8354, 4, 1), (1, 8543, 4, 2), (1, 9106, 4, 4), (1, 518, 32, 1), (1, 258, 8, 1),
    # many images, and block widths whose lanes do not fill a power of two
    (64, 1, 32, 4), (16, 1, 64, 32), (423, 5, 24, 3), (520, 3, 60, 60), (5, 2, 1560, 390), (300, 100, 488, 488), (700, 12, 488, 488),
    # stages of residual networks in 32 groups: a worker's batch
    (128, 1024, 64, 32), (128, 257, 128, 32), (64, 3137, 256, 32), (64, 785, 512, 32), (64, 196, 1024, 32), (32, 49, 2048, 32),
    (8, 4096, 64, 64), (1, 50176, 64, 32), (79, 4978, 64, 64), (2, 12688, 496, 31),
    # groups of other widths: whole images in registers
    (1, 1, 1, 1), (2, 3, 24, 2), (2, 3, 12, 4), (1, 17, 131, 1), (1, 131, 136, 8), (2, 36, 280, 1), (1, 33, 34, 2), (1, 34, 17, 1),
    (3, 65, 17, 1), (1, 65, 34, 2), (2, 130, 136, 8), (2, 132, 17, 17), (2, 132, 68, 4), (64, 196, 384, 32), (8, 1024, 640, 32),
    # and in pieces
    (1, 1, 305, 61), (3, 10, 305, 61), (1, 9, 305, 61), (2, 1, 2328, 194), (1, 2, 2104, 2), (2, 3, 1412, 4), (1, 524, 17, 1),
    (1, 283, 17, 1), (1, 67, 131, 1), (1, 130, 34, 2), (2, 40, 131, 1), (2, 3136, 256, 1), (3, 2000, 120, 1)]
