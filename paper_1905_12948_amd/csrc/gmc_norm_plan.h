// How group norm's work is laid out (gmc_norm.hip): the kernels' arguments and the
// host's choice of form, blocks and threads.  No HIP, so that it can be looked at
// without a GPU.  Not part of the ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace gmc {

constexpr int kHeldThreads = 1024;
constexpr int kHeldBlocks = 256;   // held: workgroups below which narrower blocks are tried
// backward, bytes of x from which blocks under 64 bytes wide give way to the split
// form's second read where four and more of them share a line.  In us, held and split:
// 64 x 3136 x 256 bf16 in 8-channel groups 106 and 90 (silu 125, 97), half as many
// images 54, 51, a quarter 23, 33; 16-channel groups of 512 channels (32-byte blocks)
// 199 and 196, 102 and 92, 56 and 54; f32 64 x 3136 x 128 in 4-channel groups 99 and
// 84, 32 x 6400 149 and 88.  Narrow images, whose lines few blocks share: 1024 x 3136 x
// 16 bf16 in one block 82 and 92, 200 x 8192 x 16 in two 47 and 60, 4096 x 1024 x 8
// 65 and 86, 2^19 x 8 x 8 2817 and 5446; 120 x 8192 x 32 in four 67 and 69.
constexpr int64_t kSplitBytes = int64_t(48) << 20;
constexpr int kSplitSharing = 4;
constexpr int kManyBlocks = 512;   // held: two workgroups for every CU
constexpr int kHeldMost = 16;      // vectors of x a thread holds (16 bytes each)
constexpr int kHeldMostBack = 8;   // ... of x and of dy
constexpr int kHeldChannels = 256; // threads across channels, at most
constexpr int kSplitThreads = 256;
constexpr int kSplitTile = 8;      // pixels whose loads a thread issues together
constexpr int kSplitMost = 64;     // pixels a thread sums, at most (of 2^37 values an image a few more)
constexpr int kSplitBlocks = 512;   // split: workgroups, about; long pieces stream better
                                   // (norm_back_sums at 64 x 3136 x 256: 37 us, 43 with 2048)

struct NormArgs {
    const void* x;
    const void* dy;
    void* out;  // y, or dx
    int64_t x_image, x_pixel, dy_image, dy_pixel, out_image, out_pixel;
    const float* gamma;  // NULL: ones
    const float* beta;   // NULL: zeros
    float* mean;         // [N][G]: written forward, read backward
    float* rstd;
    float* part;         // scratch
    float* part2;
    int64_t N;
    int32_t S, C, G, cpg;
    int32_t gw, cb, blocks;  // held: groups and channels per workgroup, workgroups per image
    int32_t tc, tp_log2;     // threads across channels, and the power of two above
    int32_t cpg_log2;        // -1: cpg is no power of two
    int32_t once;            // held: blocks of whole lines
    int32_t chunk, chunks;   // split: pixels per workgroup, workgroups per image
    int32_t cblocks;         // split: workgroups across channels
    float eps, inv_m;        // inv_m: 1 / (S cpg)
    int32_t act;
};

constexpr int kParamCh = 16;  // dgamma, dbeta: channels of a workgroup that sums them

inline int log2_up(int64_t n) {
    int k = 0;
    while ((int64_t(1) << k) < n) ++k;
    return k;
}

struct NormPlan {
    bool held = false;
    int vec = 1;      // channels per thread
    int threads = 0;  // held
    int kp = 0;
    int fold = 0;     // held: groups in a vector, 0: the general kernels
    size_t lds = 0;
};

// The held form for groups of a power of two of channels: whole groups in
// segments of at least `line` bytes.  Threads: as few as leave each at most 4
// vectors (forward of many blocks 8); of many blocks rather 512 threads with up to
// 16 vectors than 1024 with fewer, and for the backward pass 256 with 8 than 512,
// so that several workgroups share a CU and one loads while another computes.  64
// images of 784 pixels of 512 bf16 channels: forward 18.8 us with 512 threads, 26.6
// with 1024; 196 pixels of 1024: backward 19.3 us with 256, 23.5 with 512; one image
// of 49 pixels of 2048: forward 5.5 us with 4 vectors, 6.0 with 8.
inline bool plan_fold(NormArgs& a, NormPlan& pl, int64_t size, bool backward, int line) {
    const int full = (int)(16 / size);
    const int widest = 64 * full / a.cpg;  // groups that a block of channels may have
    for (int gw = 1; gw <= a.G && gw <= widest; ++gw) {
        if (a.G % gw) continue;
        const int64_t cb = (int64_t)gw * a.cpg;
        if (cb % full || (cb * size < line && gw < a.G)) continue;
        const int64_t tc = cb / full;
        const int lg = log2_up(tc);
        const auto vectors = [&](int threads) { return ((int64_t)a.S + (threads >> lg) - 1) / (threads >> lg); };
        const int64_t blocks = a.N * (a.G / gw);
        const int few = !backward && blocks >= kHeldBlocks ? 8 : 4;
        const int most = backward ? kHeldMostBack : kHeldMost;
        int threads = 64;
        while (threads < kHeldThreads && vectors(threads) > few) threads *= 2;
        if (blocks >= kManyBlocks) {
            if (threads == 1024 && vectors(512) <= most) threads = 512;
            if (backward && threads == 512 && vectors(256) <= most) threads = 256;
        }
        const int64_t kp = vectors(threads);
        if (kp > most) return false;
        pl.held = true;
        pl.fold = a.cpg >= full ? 1 : full / a.cpg;
        pl.vec = full;
        pl.threads = threads;
        pl.kp = (int)kp;
        a.gw = gw;
        a.cb = (int32_t)cb;
        a.blocks = a.G / gw;
        a.tc = (int32_t)tc;
        a.tp_log2 = lg;
        a.once = cb * size % 128 == 0 && (a.out_pixel * size) % 128 == 0;
        const int waves = threads / 64;
        pl.lds = sizeof(float) * (size_t)(backward ? 2 * waves * (int)cb + 2 * gw : (waves + 2) * gw);
        return true;
    }
    return false;
}

// The split form: every channel, pieces of an image.
inline NormPlan norm_plan_split(NormArgs& a, NormPlan pl, int full) {
    pl.vec = a.C % full == 0 ? full : 1;
    const int64_t vecs = a.C / pl.vec;
    a.tc = (int32_t)(vecs < kSplitThreads ? vecs : kSplitThreads);
    a.tp_log2 = log2_up(a.tc);
    a.cblocks = (int32_t)((vecs + a.tc - 1) / a.tc);
    const int rows = kSplitThreads >> a.tp_log2;
    // pixels per workgroup: enough workgroups for every CU, one to eight tiles each
    int64_t chunks = (a.S + (int64_t)rows * kSplitTile - 1) / ((int64_t)rows * kSplitTile);
    const int64_t want = (kSplitBlocks + a.N * a.cblocks - 1) / (a.N * a.cblocks);
    const int64_t least = (a.S + (int64_t)rows * kSplitMost - 1) / ((int64_t)rows * kSplitMost);
    if (chunks > want) chunks = want > least ? want : least;
    const int64_t most = 0x7fffffff / a.C;  // norm_join counts an image's chunks and channels in 32 bits
    if (chunks > most) chunks = most;
    a.chunk = (int32_t)((a.S + chunks - 1) / chunks);
    a.chunks = (int32_t)(((int64_t)a.S + a.chunk - 1) / a.chunk);
    const int slots = a.tp_log2 < 6 ? kSplitThreads / 64 : rows;
    pl.threads = kSplitThreads;
    pl.lds = sizeof(float) * ((size_t)(slots + 1) * pl.vec << a.tp_log2);
    return pl;
}

// Chooses the form and fills the geometry of a; size: bytes of an element.
inline NormPlan norm_plan(NormArgs& a, int64_t size, bool backward) {
    NormPlan pl;
    const int full = (int)(16 / size);
    const int most = backward ? kHeldMostBack : kHeldMost;
    a.cpg = a.C / a.G;
    a.inv_m = (float)(1.0 / ((double)a.S * (double)a.cpg));
    a.cpg_log2 = a.cpg & (a.cpg - 1) ? -1 : log2_up(a.cpg);
    if (a.cpg_log2 >= 0 && a.cpg <= 64) {
        for (int line = 128; line >= 16; line >>= 1) {
            if (!plan_fold(a, pl, size, backward, line)) continue;
            if (a.N * a.blocks >= kHeldBlocks) break;
        }
        if (pl.held && !(backward && (int64_t)a.cb * size < 64 && a.blocks >= kSplitSharing &&
                         a.N * (int64_t)a.S * a.C * size >= kSplitBytes)) return pl;
        if (pl.held) {
            pl = NormPlan{};
            return norm_plan_split(a, pl, full);
        }
    }
    // any groups: the fewest whose channels fill a 128-byte line (else a 64-byte
    // half), with a thread count that leaves at most `most` vectors each
    const int widest = kHeldChannels * full / a.cpg;
    for (int line = 128; line >= 64 && !pl.held; line >>= 1)
        for (int gw = 1; gw <= a.G && gw <= widest && !pl.held; ++gw) {
            if (a.G % gw) continue;
            const int64_t cb = (int64_t)gw * a.cpg;
            const bool wide = cb * size >= line;
            if (!wide && gw < a.G) continue;
            const int vec = cb % full == 0 ? full : 1;
            const int64_t tc = cb / vec;
            if (tc > kHeldChannels) continue;
            const int lg = log2_up(tc);
            int threads = 256;
            while (threads < kHeldThreads && (((int64_t)a.S << lg) + threads - 1) / threads > 4) threads *= 2;
            const int rows = threads >> lg;
            const int64_t kp = ((int64_t)a.S + rows - 1) / rows;
            if (kp > most) continue;
            pl.held = true;
            pl.vec = vec;
            pl.threads = threads;
            pl.kp = kp <= 4 ? 4 : most;
            a.gw = gw;
            a.cb = (int32_t)cb;
            a.blocks = a.G / gw;
            a.tc = (int32_t)tc;
            a.tp_log2 = lg;
            const int slots = lg < 6 ? threads / 64 : rows;
            pl.lds = sizeof(float) * (((size_t)(slots + 1) * vec << lg) + 2 * (size_t)gw);
        }
    if (pl.held) return pl;
    return norm_plan_split(a, pl, full);
}

// Scratch in floats: two arrays of per-channel partial values, and for the
// split backward pass the two shared terms of every group.
inline int64_t norm_scratch(const NormArgs& a, const NormPlan& pl, bool backward) {
    if (pl.held) return backward ? 2 * a.N * a.C : 0;
    return 2 * a.N * a.chunks * a.C + (backward ? 2 * a.N * a.G : 0);
}

constexpr int64_t kMostThreads = 0xffffffffll;  // of one launch

inline unsigned param_blocks(int32_t C) { return (unsigned)(((int64_t)C + kParamCh - 1) / kParamCh); }

// Images one launch of each kernel may have; a call of more takes several.
inline int64_t launch_images(const NormArgs& a, const NormPlan& pl, bool backward) {
    const int64_t params = backward ? param_blocks(a.C) * (int64_t)kSplitThreads : 0;
    if (params >= kMostThreads) return 0;
    if (pl.held) return kMostThreads / (pl.threads * (int64_t)a.blocks);
    const int64_t pieces = (kMostThreads - params) / (kSplitThreads * (int64_t)a.chunks * a.cblocks);
    const int64_t joins = kMostThreads / 64 / a.G;
    return pieces < joins ? pieces : joins;
}

}  // namespace gmc
