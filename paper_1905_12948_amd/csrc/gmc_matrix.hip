// Orthogonalised matrices of a flat vector (gmc_orthogonalize and
// gmc_orthogonal_step in include/gmc.h): Newton-Schulz steps
//   X <- a X + (b G + c G G) X,  G = X X^T,
// from X = M / (|M| + eps), |.| the Frobenius norm, M taken on its side where it
// has more rows than columns (the steps commute with transposition): X is m x n,
// m <= n.
//
// Precision.  The steps amplify small singular values by up to prod a_k (485 for
// the five usual ones) and with them any rounding of X, so X, G and the polynomial
// are kept to 22 bits: each value as the sum of two halves, hi = f16(v) and lo =
// f16(v - hi), v the value times a power of two that keeps lo clear of the smallest
// f16 (X and G: 2^13, the polynomial: 2^10).  A product is hi hi + hi lo + lo hi on the f16
// matrix instructions with sums in 32 bits: what is left out, lo lo, is 2^-22 of it.  The
// result is as near to the 64-bit one as products in 32 bits are.
//
// Where |M| is not far above eps X is small, as small as M, and would leave f16's range: what
// is held is Y = X / theta, theta <= 1 a number of the matrix and the step: at first
// |M| / (|M| + eps), so that |Y| = 1, then as much more as the step's polynomial can
// amplify, up to 1.  In Y a step is Y <- (theta / theta') (a Y + (b theta^2 G + c theta^4 G G) Y).
//
// Layout.  X (along n), its transpose (along m), G and the polynomial are stored in
// the order the matrix instructions read: blocks of 32 rows x 16 columns, lane l's
// eight neighbours of row l % 32 as 16 bytes at l * 16, hi then lo.  Every operand is
// read along its contraction (X for G; G, which is its own transpose; X^T for the
// last product), so a tile's blocks go to shared memory and to registers in whole
// kilobytes, with no bank conflict and no swizzle.  Rows and columns are padded with
// zeros to 32, which the steps keep.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "gmc_ops.h"

namespace gmc {

namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kScaleX = 0x1p13f, kScaleB = 0x1p10f;   // of X and G, and of b G + c G^2
constexpr int kSide = 64;                                // side of the pieces the vector is read in
constexpr int kParts = 256;                              // partial sums of a matrix's squares
constexpr int64_t kGapChunk = 8192;                      // components outside the matrices, a workgroup
constexpr int kMostSteps = 64;

// A matrix of the plan.  m <= n are its sides, mb and nb their number in blocks of 32.
struct Mat {
    int64_t offset, pitch;
    int64_t x, g;      // first block of X (and of X^T) and of G
    int32_t rows, cols, m, n, mb, nb;
    int32_t flip;      // rows > cols: X is the transpose
    float scale;
    int32_t part, parts;
};

struct Tile {
    int32_t mat, i, j, count;
};

struct Gap {
    int64_t at, len;
};

// -- the vector in and out --------------------------------------------------------

struct VectorArgs {
    const Mat* mats;
    const Tile* tiles;
    const void* x;      // the vector, or the step's update
    float* momentum;    // NULL: none
    float mu;
    int32_t nesterov;
    double* part;
    double eps;
    _Float16 *X, *XT;
    float* theta;              // [matrices][kMostSteps + 1]
    int32_t steps;
    float growth[kMostSteps];  // by which a step amplifies at most, 1 or more
};

// What is orthogonalised, from the update and the momentum that holds it already.
__device__ __forceinline__ float direction(const VectorArgs& a, float u, float v) { return a.nesterov ? u + a.mu * v : v; }

// Sums of squares in 64 bits (no 32-bit value's square leaves their range), and the
// momentum's update on the way.  A tile of the launch is `count` pieces of a matrix.
template <int DT, bool kStep>
__global__ __launch_bounds__(256) void matrix_norm(VectorArgs a) {
    typedef typename Elem<DT>::T T;
    __shared__ double lds[4];
    const Tile t = a.tiles[blockIdx.x];
    const Mat m = a.mats[t.mat];
    const T* x = static_cast<const T*>(a.x) + m.offset;
    const int wide = (m.cols + kSide - 1) / kSide;
    const int r0 = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * 4;
    double sum = 0.0;
    for (int k = 0; k < t.count; ++k) {
        const int piece = t.i + k, pr = piece / wide, pc = piece - pr * wide;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t r = (int64_t)pr * kSide + r0 + 16 * q;
            const int c = pc * kSide + c0;
            if (r >= m.rows || c >= m.cols) continue;
            const int64_t at = r * m.pitch + c;
            const int n = m.cols - c < 4 ? m.cols - c : 4;
            float u[4] = {};
            if (n == 4) {
                Vec<DT, DT == GMC_F32 ? 4 : 2> v0, v1;
                if constexpr (DT == GMC_F32) {
                    v0 = Vec<DT, 4>::load(x + at);
                    v0.unpack(u);
                } else {
                    v0 = Vec<DT, 2>::load(x + at);
                    v1 = Vec<DT, 2>::load(x + at + 2);
                    float p[2];
                    v0.unpack(p);
                    u[0] = p[0], u[1] = p[1];
                    v1.unpack(p);
                    u[2] = p[0], u[3] = p[1];
                }
            } else {
                for (int e = 0; e < n; ++e) u[e] = Elem<DT>::up(x[at + e]);
            }
            if constexpr (kStep) {
                if (a.momentum) {
                    float* v = a.momentum + m.offset + at;
                    float w[4] = {};
                    if (n == 4) Vec<GMC_F32, 4>::load(v).unpack(w);
                    else
                        for (int e = 0; e < n; ++e) w[e] = v[e];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = a.mu * w[e] + u[e];
                        u[e] = direction(a, u[e], w[e]);
                    }
                    if (n == 4) {
                        Vec<GMC_F32, 4> o;
                        o.pack(w);
                        o.store(v);
                    } else {
                        for (int e = 0; e < n; ++e) v[e] = w[e];
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) sum += (double)u[e] * (double)u[e];
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.part[m.part + t.j] = lds[0] + lds[1] + lds[2] + lds[3];
}

// A value as its two halves.
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// The matrix over its norm, in halves, along both of its axes.
template <int DT, bool kStep>
__global__ __launch_bounds__(256) void matrix_pack(VectorArgs a) {
    typedef typename Elem<DT>::T T;
    __shared__ float in[kSide][kSide + 1];
    __shared__ double lds[4];
    const Tile t = a.tiles[blockIdx.x];
    const Mat m = a.mats[t.mat];
    const T* x = static_cast<const T*>(a.x) + m.offset;
    double sum = (int)threadIdx.x < m.parts ? a.part[m.part + threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    // piece (i, j) of X is piece (j, i) of a matrix on its side
    const int pr = m.flip ? t.j : t.i, pc = m.flip ? t.i : t.j;
    const int c0 = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const int r0 = (threadIdx.x >> 6) + 4 * q;
        const int64_t r = (int64_t)pr * kSide + r0;
        const int c = pc * kSide + c0;
        float u = 0.0f;
        if (r < m.rows && c < m.cols) {
            const int64_t at = r * m.pitch + c;
            u = Elem<DT>::up(x[at]);
            if constexpr (kStep)
                if (a.momentum) u = direction(a, u, a.momentum[m.offset + at]);
        }
        in[r0][c0] = u;
    }
    __syncthreads();
    const double norm = sqrt(lds[0] + lds[1] + lds[2] + lds[3]);
    const double inv = norm == 0.0 ? 0.0 : (double)kScaleX / norm;
    if (t.i == 0 && t.j == 0 && threadIdx.x == 0) {
        float v = norm == 0.0 ? 1.0f : (float)(norm / (norm + a.eps));
        float* theta = a.theta + t.mat * (kMostSteps + 1);
        theta[0] = v;
        for (int k = 0; k < a.steps; ++k) theta[k + 1] = v = fminf(v * a.growth[k], 1.0f) + 0.0f * v;   // NaN stays
    }
    const int64_t kn = 2 * (int64_t)m.nb, km = 2 * (int64_t)m.mb;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        // eight neighbours: of X's rows (u < 2) or of its columns
        const int unit = threadIdx.x + 256 * (u & 1), row = unit & 63, k8 = unit >> 6;
        const bool along = u < 2;
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = along ? row : 8 * k8 + e, j = along ? 8 * k8 + e : row;
            _Float16 h, l;
            split((float)((double)(m.flip ? in[j][i] : in[i][j]) * inv), h, l);
            hi[e] = h;
            lo[e] = l;
        }
        const int rb = (along ? t.i : t.j) * 2 + (row >> 5), kb = (along ? t.j : t.i) * 4 + (k8 >> 1);
        if (rb < (along ? m.mb : m.nb) && kb < (along ? kn : km)) {
            _Float16* o = (along ? a.X : a.XT) + (m.x + rb * (along ? kn : km) + kb) * 1024 + ((row & 31) + 32 * (k8 & 1)) * 8;
            *reinterpret_cast<f16x8*>(o) = hi;
            *reinterpret_cast<f16x8*>(o + 512) = lo;
        }
    }
}

// Components outside the matrices: out = x, or w + update.
template <int DT, bool kStep>
__global__ __launch_bounds__(256) void matrix_gaps(const Gap* gaps, const void* in, const float* w, void* out) {
    typedef typename Elem<DT>::T T;
    const Gap g = gaps[blockIdx.x];
    const T* x = static_cast<const T*>(in) + g.at;
    for (int64_t i = threadIdx.x; i < g.len; i += 256) {
        if constexpr (kStep) static_cast<float*>(out)[g.at + i] = w[g.at + i] + Elem<DT>::up(x[i]);
        else static_cast<T*>(out)[g.at + i] = x[i];
    }
}

// -- products ---------------------------------------------------------------------

enum { kGram, kPoly, kApply, kLast, kLastStep };

struct ProductArgs {
    const Mat* mats;
    const Tile* tiles;
    const _Float16 *X, *XT, *G, *B;  // what the mode reads
    _Float16 *Xo, *XTo, *Go, *Bo;    // and writes
    const float* theta;  // this step's of the first matrix
    float a, b, c;
    void* out;        // kLast, kLastStep
    const float* w;   // kLastStep
    float alpha, keep;
};

// Waits until all but the wavefront's last kLoads loads to shared memory have arrived and its
// reads of shared memory are done, and then for the workgroup's other wavefronts.
template <int kLoads>
__device__ __forceinline__ void wait_stage() {
    static_assert(kLoads < 64, "the counter has 6 bits");
    __builtin_amdgcn_s_waitcnt((kLoads & 15) | 7 << 4 | 0 << 8 | (kLoads >> 4) << 14);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// One tile of D = P Q^T, both along their contraction, by four wavefronts of kWide x
// kWide blocks each, and what the mode makes of it:
//   kGram   P = Q = X            G = D
//   kPoly   P = Q = G            B = b G + c D
//   kApply  P = B, Q = X^T       X <- a X + D, along both axes
//   kLast   the same, or P = X^T and Q = B for a matrix on its side, into the vector
// G and B are symmetric: tiles with j <= i, written to both places.
template <int kWide, int kMode, int DT>
__global__ __launch_bounds__(256, 2) void matrix_product(ProductArgs a) {
    constexpr int kBlocks = 2 * kWide;                 // of 32 rows, on each side of the tile
    constexpr int kDeep = kWide == 2 ? 1 : 2;          // 16 columns, of a stage
    constexpr int kChunks = 2 * kBlocks * kDeep * 2;   // kilobytes of a stage: sides, blocks, columns, halves
    __shared__ _Float16 stage0[kChunks * 512], stage1[kChunks * 512], stage2[kChunks * 512], stage3[kChunks * 512];
    const Tile t = a.tiles[blockIdx.x];
    const Mat m = a.mats[t.mat];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const bool last = kMode == kLast || kMode == kLastStep;
    const bool flip = last && m.flip;
    const int ti = flip ? t.j : t.i, tj = flip ? t.i : t.j;
    const _Float16* P = (kMode == kGram ? a.X + m.x * 1024 : kMode == kPoly ? a.G + m.g * 1024
                         : flip ? a.XT + m.x * 1024 : a.B + m.g * 1024);
    const _Float16* Q = (kMode == kGram ? a.X + m.x * 1024 : kMode == kPoly ? a.G + m.g * 1024
                         : flip ? a.B + m.g * 1024 : a.XT + m.x * 1024);
    const int pb = kMode == kGram || kMode == kPoly ? m.mb : flip ? m.nb : m.mb;   // blocks of P's and Q's rows
    const int qb = kMode == kGram || kMode == kPoly ? m.mb : flip ? m.mb : m.nb;
    const int deep = 2 * (kMode == kGram ? m.nb : m.mb);   // 16 columns
    const int64_t row = (int64_t)deep * 1024;              // halves of a row of blocks
    const float theta = kMode == kGram ? 1.0f : a.theta[t.mat * (kMostSteps + 1)];
    const float ratio = kMode == kApply ? theta / a.theta[t.mat * (kMostSteps + 1) + 1] : 1.0f;

    // chunk c of a stage: side, block, 16 columns, half; a wavefront takes every fourth.
    // Blocks beyond the matrix are read as its last one and not written.
    const _Float16* from[kChunks / 4];
#pragma unroll
    for (int k = 0; k < kChunks / 4; ++k) {
        const int c = k * 4 + wave, side = c / (kChunks / 2), b = c / (2 * kDeep) % kBlocks;
        int rb = (side ? tj : ti) * kBlocks + b;
        const int most = (side ? qb : pb) - 1;
        rb = rb < most ? rb : most;
        from[k] = (side ? Q : P) + rb * row + (c % (2 * kDeep)) * 512 + lane * 8;
    }
    f32x16 acc[kWide][kWide];
#pragma unroll
    for (int i = 0; i < kWide; ++i)
#pragma unroll
        for (int j = 0; j < kWide; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    const int wi = (wave >> 1) * kWide, wj = (wave & 1) * kWide;   // the wavefront's first blocks
    const int stages = deep / kDeep;
    const auto fetch = [&](int s, _Float16* to) {
        s = s < stages ? s : stages - 1;   // the count of loads under way stays what the waits take it for
#pragma unroll
        for (int k = 0; k < kChunks / 4; ++k)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from[k] + (int64_t)s * (kDeep * 1024)),
                                             (__attribute__((address_space(3))) void*)(to + (k * 4 + wave) * 512), 16, 0, 0);
    };
    // Stage s is in shared memory and stage s - 1 has been read by all, whose place the loads of
    // s + 3 take; those of s + 1 and s + 2 stay under way.
    const auto step = [&](int s, const _Float16* here, _Float16* next) {
        wait_stage<2 * (kChunks / 4)>();
        const f16x8* at = reinterpret_cast<const f16x8*>(here) + lane;
        f16x8 p[kDeep][kWide][2], q[kDeep][kWide][2];
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kWide; ++i) {
                    p[k][i][h] = at[(((wi + i) * kDeep + k) * 2 + h) * 64];
                    q[k][i][h] = at[(((kBlocks + wj + i) * kDeep + k) * 2 + h) * 64];
                }
        fetch(s + 3, next);
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
#pragma unroll
            for (int part = 0; part < 3; ++part)
#pragma unroll
                for (int i = 0; i < kWide; ++i)
#pragma unroll
                    for (int j = 0; j < kWide; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[k][i][part == 2], q[k][j][part == 1], acc[i][j], 0, 0, 0);
    };
    fetch(0, stage0);
    fetch(1, stage1);
    fetch(2, stage2);
    int s = 0;
    for (; s + 4 <= stages; s += 4) {
        step(s, stage0, stage3);
        step(s + 1, stage1, stage0);
        step(s + 2, stage2, stage1);
        step(s + 3, stage3, stage2);
    }
    if (s < stages) step(s, stage0, stage3);
    if (s + 1 < stages) step(s + 1, stage1, stage0);
    if (s + 2 < stages) step(s + 2, stage2, stage1);
    __syncthreads();   // no load is under way and shared memory is free

    // Of a block of D lane l has column l % 32, rows 8 g + 4 (l / 32) + e in entry 4 g + e.
    static_assert(32 * 33 * 4 <= kChunks * 1024, "a wavefront's block fits a stage");
    float* turn = reinterpret_cast<float*>(wave == 0 ? stage0 : wave == 1 ? stage1 : wave == 2 ? stage2 : stage3);
    const int col = lane & 31, half = lane >> 5;
#pragma unroll
    for (int i = 0; i < kWide; ++i)
#pragma unroll
        for (int j = 0; j < kWide; ++j) {
            const int ib = ti * kBlocks + wi + i, jb = tj * kBlocks + wj + j;
            if (ib >= pb || jb >= qb) continue;
            f32x16 d = acc[i][j];
            // entry (i, j) where its row is j: block (jb, 2 ib + g / 2), lane col + 32 (g % 2), halves 4 half + e
            const int64_t place = ((int64_t)jb * 2 * pb + 2 * ib) * 1024 + col * 8 + 4 * half;
            if constexpr (kMode == kGram) {
#pragma unroll
                for (int e = 0; e < 16; ++e) d[e] *= 1.0f / kScaleX;
            } else {
                // d <- u (hi + lo) + v d
                const float u = kMode == kPoly ? a.b * (theta * theta) * (kScaleB / kScaleX) : a.a * ratio;
                const float v = kMode == kPoly ? a.c * (theta * theta) * (theta * theta) * (kScaleB / kScaleX / kScaleX) : ratio / kScaleB;
                const _Float16* add = (kMode == kPoly ? a.G + m.g * 1024 : flip ? a.X + m.x * 1024 : a.XT + m.x * 1024) + place;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f16x4 hi = *reinterpret_cast<const f16x4*>(add + (g >> 1) * 1024 + (g & 1) * 256);
                    const f16x4 lo = *reinterpret_cast<const f16x4*>(add + (g >> 1) * 1024 + (g & 1) * 256 + 512);
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[4 * g + e] = u * ((float)hi[e] + (float)lo[e]) + v * d[4 * g + e];
                }
            }
            if constexpr (last) {
                typedef typename Elem<DT>::T T;
                const float factor = a.alpha * m.scale * theta * (1.0f / kScaleX);
                const int c = jb * 32 + col;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = ib * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                    if (r >= m.rows || c >= m.cols) continue;
                    const int64_t at = m.offset + (int64_t)r * m.pitch + c;
                    if constexpr (kMode == kLastStep) static_cast<float*>(a.out)[at] = a.keep * a.w[at] + factor * d[e];
                    else static_cast<T*>(a.out)[at] = Elem<DT>::down(factor * d[e]);
                }
                continue;
            }
            _Float16* o = (kMode == kGram ? a.Go + m.g * 1024 : kMode == kPoly ? a.Bo + m.g * 1024 : a.XTo + m.x * 1024) + place;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f16x4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    _Float16 h, l;
                    split(d[4 * g + e], h, l);
                    hi[e] = h;
                    lo[e] = l;
                }
                *reinterpret_cast<f16x4*>(o + (g >> 1) * 1024 + (g & 1) * 256) = hi;
                *reinterpret_cast<f16x4*>(o + (g >> 1) * 1024 + (g & 1) * 256 + 512) = lo;
            }
            if (kMode != kApply && ti == tj) continue;
            // and where its row is i, through shared memory of the wavefront's own
#pragma unroll
            for (int e = 0; e < 16; ++e) turn[(8 * (e >> 2) + 4 * half + (e & 3)) * 33 + col] = d[e];
            __builtin_amdgcn_wave_barrier();
            o = (kMode == kGram ? a.Go + m.g * 1024 : kMode == kPoly ? a.Bo + m.g * 1024 : a.Xo + m.x * 1024) +
                ((int64_t)ib * 2 * qb + 2 * jb) * 1024 + lane * 8;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                f16x8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    _Float16 h, l;
                    split(turn[col * 33 + 16 * k + 8 * half + e], h, l);
                    hi[e] = h;
                    lo[e] = l;
                }
                *reinterpret_cast<f16x8*>(o + k * 1024) = hi;
                *reinterpret_cast<f16x8*>(o + k * 1024 + 512) = lo;
            }
            __builtin_amdgcn_wave_barrier();
        }
}

}  // namespace

}  // namespace gmc

using namespace gmc;

// The plan: the matrices, and which tile of which matrix each workgroup of a launch takes.
struct gmc_matrices {
    int64_t d = 0;
    int device = 0;
    int wide = 1;              // blocks a wavefront's side of a tile
    int32_t n = 0;
    int64_t blocks_x = 0, blocks_g = 0, parts = 0;
    int64_t norms = 0, pieces = 0, grams = 0, applies = 0, gaps = 0;
    void* table = nullptr;     // device memory: all of the below
    const Mat* mats = nullptr;
    const Tile *norm = nullptr, *pack = nullptr, *gram = nullptr, *apply = nullptr;
    const Gap* gap = nullptr;
};

namespace gmc {

namespace {

constexpr int64_t kMostTiles = int64_t(1) << 22;

int64_t up_to(int64_t v, int64_t step) { return (v + step - 1) / step; }

// Whether the matrices share no component: sorted by offset, neighbours are apart, or are
// column slices of one wide array (rows the same distance apart, columns apart).
struct Part {
    int64_t offset, rows, cols, pitch;
    int64_t end() const { return offset + (rows - 1) * pitch + cols; }
};

bool disjoint(std::vector<Part> p) {
    std::sort(p.begin(), p.end(), [](const Part& a, const Part& b) { return a.offset < b.offset; });
    for (size_t i = 0; i < p.size(); ++i)
        for (size_t k = i + 1; k < p.size() && p[k].offset < p[i].end(); ++k) {
            if (p[k].pitch != p[i].pitch || p[i].rows == 1 || p[k].rows == 1) {
                // a single row between two rows of the other
                const Part &one = p[i].rows == 1 ? p[i] : p[k], &more = p[i].rows == 1 ? p[k] : p[i];
                if (one.rows != 1 || p[i].rows == 1) return false;
                const int64_t c = (one.offset - more.offset) % more.pitch;
                if (c < more.cols || c + one.cols > more.pitch) return false;
                continue;
            }
            const int64_t c = (p[k].offset - p[i].offset) % p[i].pitch;
            if (c < p[i].cols || c + p[k].cols > p[i].pitch) return false;
        }
    return true;
}

// The largest |x| and |b x^2 + c x^4| that singular values in [0, top] are taken to,
// or a negative number where one is not finite.
struct Reach {
    double x, poly, growth;   // growth: the largest |a + b x^2 + c x^4|
};

Reach reach(double a, double b, double c, double top) {
    const auto p = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
    const auto q = [&](double s) { return fabs(s * s * (b + s * s * c)); };
    // extrema inside: 5 c y^2 + 3 b y + a = 0 and 2 c y + b = 0 in y = s^2
    double y[3] = {-1.0, -1.0, -1.0};
    if (c != 0.0) {
        const double r = 9.0 * b * b - 20.0 * a * c;
        if (r >= 0.0) {
            y[0] = (-3.0 * b + sqrt(r)) / (10.0 * c);
            y[1] = (-3.0 * b - sqrt(r)) / (10.0 * c);
        }
        y[2] = -b / (2.0 * c);
    } else if (b != 0.0) {
        y[0] = -a / (3.0 * b);
    }
    const auto slope = [&](double s) { return fabs(a + s * s * (b + s * s * c)); };
    Reach m = {p(top), q(top), fmax(fabs(a), slope(top))};
    for (double v : y) {
        const double s = v > 0.0 ? sqrt(v) : 0.0;
        if (s < top) {
            m.x = fmax(m.x, p(s));
            m.poly = fmax(m.poly, q(s));
            m.growth = fmax(m.growth, slope(s));
        }
    }
    if (!isfinite(m.x) || !isfinite(m.poly)) m.x = m.poly = INFINITY;
    return m;
}

struct Scratch {
    _Float16 *X, *T0, *T1, *G, *B;
    double* part;
    float* theta;
    int64_t bytes;
};

Scratch layout(const gmc_matrices* p, void* base) {
    char* at = static_cast<char*>(base);
    Scratch s;
    const auto take = [&](int64_t bytes) {
        char* here = at;
        at += up_to(bytes, 256) * 256;
        return here;
    };
    s.X = reinterpret_cast<_Float16*>(take(p->blocks_x * 2048));
    s.T0 = reinterpret_cast<_Float16*>(take(p->blocks_x * 2048));
    s.T1 = reinterpret_cast<_Float16*>(take(p->blocks_x * 2048));
    s.G = reinterpret_cast<_Float16*>(take(p->blocks_g * 2048));
    s.B = reinterpret_cast<_Float16*>(take(p->blocks_g * 2048));
    s.part = reinterpret_cast<double*>(take(p->parts * 8));
    s.theta = reinterpret_cast<float*>(take((int64_t)p->n * (kMostSteps + 1) * 4));
    s.bytes = at - static_cast<char*>(base);
    return s;
}

// What both calls refuse.
gmc_status matrices_check(const char* me, const gmc_matrices* p, int32_t dtype, int32_t steps, const double* coefficients,
                          double eps, const void* workspace, int64_t workspace_bytes) {
    if (!p) return op_error(GMC_EINVAL, me, "NULL argument");
    if (!known_type(dtype)) return op_error(GMC_EINVAL, me, "unknown element type");
    if (steps < 1 || steps > kMostSteps || !coefficients) return op_error(GMC_EINVAL, me, "need coefficients of 1 to 64 steps");
    if (!(eps >= 0.0 && eps <= 1.0)) return op_error(GMC_EINVAL, me, "eps must be in [0, 1]");
    double top = 1.0;
    for (int32_t k = 0; k < steps; ++k) {
        const double *c = coefficients + 3 * k;
        if (!isfinite(c[0]) || !isfinite(c[1]) || !isfinite(c[2])) return op_error(GMC_EINVAL, me, "a coefficient is not finite");
        const Reach r = reach(c[0], c[1], c[2], top);
        // X and G by 2^13 and the polynomial by 2^10 have to stay below f16's 65504
        if (!(r.x <= 2.5 && r.poly <= 60.0) && !(k == steps - 1 && r.x <= 1e6 && r.poly <= 60.0))
            return op_error(GMC_EINVAL, me, "the coefficients take a singular value beyond 2.5");
        top = r.x;
    }
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess) return op_error(GMC_EDEVICE, me, "no current device");
    if (device != p->device) return op_error(GMC_EINVAL, me, "the plan is another device's");
    if (p->n) {
        if (!workspace || workspace_bytes < gmc_matrices_workspace(p)) return op_error(GMC_EINVAL, me, "the workspace is too small");
        if (reinterpret_cast<uintptr_t>(workspace) & 255u) return op_error(GMC_EINVAL, me, "the workspace is not 256-byte aligned");
    }
    return GMC_OK;
}

struct Steps {
    int32_t n;
    const double* coefficients;
    double eps;
};

template <int DT, bool kStep, int kWide>
void run_products(const gmc_matrices* p, const Scratch& s, const Steps& how, ProductArgs a, hipStream_t st) {
    const dim3 grams((unsigned)p->grams), applies((unsigned)p->applies);
    _Float16 *from = s.T0, *to = s.T1;
    for (int32_t k = 0; k < how.n; ++k) {
        a.a = (float)how.coefficients[3 * k];
        a.b = (float)how.coefficients[3 * k + 1];
        a.c = (float)how.coefficients[3 * k + 2];
        a.X = s.X;
        a.Xo = s.X;
        a.G = a.Go = s.G;
        a.B = a.Bo = s.B;
        a.XT = from;
        a.XTo = to;
        a.theta = s.theta + k;
        a.tiles = p->gram;
        matrix_product<kWide, kGram, GMC_F32><<<grams, 256, 0, st>>>(a);
        matrix_product<kWide, kPoly, GMC_F32><<<grams, 256, 0, st>>>(a);
        a.tiles = p->apply;
        if (k + 1 < how.n) matrix_product<kWide, kApply, GMC_F32><<<applies, 256, 0, st>>>(a);
        else if (kStep) matrix_product<kWide, kLastStep, GMC_F32><<<applies, 256, 0, st>>>(a);
        else matrix_product<kWide, kLast, DT><<<applies, 256, 0, st>>>(a);
        std::swap(from, to);
    }
}

template <int DT, bool kStep>
void run_steps(const gmc_matrices* p, const Scratch& s, const Steps& how, const VectorArgs& v, const ProductArgs& a, hipStream_t st) {
    VectorArgs n = v;
    n.mats = p->mats;
    n.tiles = p->norm;
    n.part = s.part;
    n.eps = how.eps;
    n.theta = s.theta;
    n.steps = how.n;
    double top = 1.0;
    for (int32_t k = 0; k < how.n; ++k) {
        const Reach r = reach(how.coefficients[3 * k], how.coefficients[3 * k + 1], how.coefficients[3 * k + 2], top);
        n.growth[k] = (float)fmax(r.growth, 1.0);
        top = r.x;
    }
    n.X = s.X;
    n.XT = s.T0;
    matrix_norm<DT, kStep><<<dim3((unsigned)p->norms), 256, 0, st>>>(n);
    n.tiles = p->pack;
    matrix_pack<DT, kStep><<<dim3((unsigned)p->pieces), 256, 0, st>>>(n);
    if (p->wide == 2) run_products<DT, kStep, 2>(p, s, how, a, st);
    else run_products<DT, kStep, 1>(p, s, how, a, st);
}

}  // namespace

}  // namespace gmc

extern "C" {

gmc_status gmc_matrices_init(gmc_matrices** out, int64_t d, int32_t n, const int64_t* offset, const int64_t* rows,
                             const int64_t* cols, const int64_t* pitch, const double* scale) {
    const char* me = "gmc_matrices_init";
    if (!out) return op_error(GMC_EINVAL, me, "NULL argument");
    *out = nullptr;
    if (d < 1 || d > (int64_t(1) << 40)) return op_error(GMC_EINVAL, me, "need 1 <= d <= 2^40");
    if (n < 0 || n > 8192) return op_error(GMC_EINVAL, me, "need 0 to 8192 matrices");
    if (n && (!offset || !rows || !cols)) return op_error(GMC_EINVAL, me, "NULL argument");
    gmc_matrices* p = nullptr;
    try {
        std::vector<Part> parts;
        for (int32_t k = 0; k < n; ++k) {
            const Part q = {offset[k], rows[k], cols[k], pitch ? pitch[k] : cols[k]};
            constexpr int64_t kMost = int64_t(1) << 26;
            if (q.rows < 1 || q.cols < 1 || q.rows > kMost || q.cols > kMost)
                return op_error(GMC_EINVAL, me, "a matrix needs 1 to 2^26 rows and columns");
            if (q.pitch < q.cols || q.pitch > d) return op_error(GMC_EINVAL, me, "a pitch is shorter than a row, or longer than the vector");
            if (q.offset < 0 || q.offset >= d || (q.rows > 1 && q.rows - 1 > d / q.pitch) || q.end() > d)
                return op_error(GMC_EINVAL, me, "a matrix does not lie inside the vector");
            if (scale && !(fabs(scale[k]) <= 3.0e38)) return op_error(GMC_EINVAL, me, "a scale is not finite in fp32");
            parts.push_back(q);
        }
        if (!disjoint(parts)) return op_error(GMC_EINVAL, me, "two matrices share components");
        p = new gmc_matrices;
        p->d = d;
        p->n = n;
        std::vector<Mat> mats;
        int64_t large = 0;
        for (int32_t k = 0; k < n; ++k) {
            const Part& q = parts[k];
            Mat m{};
            m.offset = q.offset;
            m.pitch = q.pitch;
            m.rows = (int32_t)q.rows;
            m.cols = (int32_t)q.cols;
            m.flip = q.rows > q.cols;
            m.m = m.flip ? m.cols : m.rows;
            m.n = m.flip ? m.rows : m.cols;
            m.mb = (m.m + 31) / 32;
            m.nb = (m.n + 31) / 32;
            m.scale = scale ? (float)scale[k] : 1.0f;
            m.x = p->blocks_x;
            m.g = p->blocks_g;
            p->blocks_x += (int64_t)m.mb * m.nb * 2;
            p->blocks_g += (int64_t)m.mb * m.mb * 2;
            large += up_to(m.mb, 4) * up_to(m.nb, 4);
            mats.push_back(m);
        }
        p->wide = large >= 256 ? 2 : 1;
        const int side = 2 * p->wide;
        std::vector<Tile> norm, pack, gram, apply;
        std::vector<int32_t> order(n);
        for (int32_t k = 0; k < n; ++k) order[k] = k;
        // the longest contractions first: they end last
        std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return mats[x].n > mats[y].n; });
        bool many = false;
        for (int32_t o = 0; o < n && !many; ++o) {
            const int32_t k = order[o];
            Mat& m = mats[k];
            const int64_t mt = up_to(m.mb, side), nt = up_to(m.nb, side), mp = up_to(m.m, kSide), np = up_to(m.n, kSide);
            if (mt > kMostTiles / nt || mp > kMostTiles / np) {
                many = true;
                break;
            }
            const int64_t each = up_to(mp * np, kParts);
            m.parts = (int32_t)up_to(mp * np, each);
            m.part = (int32_t)p->parts;
            p->parts += m.parts;
            for (int32_t q = 0; q < m.parts; ++q)
                norm.push_back({k, (int32_t)(q * each), q, (int32_t)std::min(each, mp * np - q * each)});
            for (int32_t i = 0; i < mp; ++i)
                for (int32_t j = 0; j < np; ++j) pack.push_back({k, i, j, 0});
            for (int32_t i = 0; i < mt; ++i)
                for (int32_t j = 0; j <= i; ++j) gram.push_back({k, i, j, 0});
            for (int32_t i = 0; i < mt; ++i)
                for (int32_t j = 0; j < nt; ++j) apply.push_back({k, i, j, 0});
            many = (int64_t)std::max(pack.size(), apply.size()) > kMostTiles;
        }
        if (many) {
            delete p;
            return op_error(GMC_EINVAL, me, "more than 2^22 tiles");
        }
        // components between the matrices' rows
        std::vector<std::pair<int64_t, int64_t>> spans;
        for (const Part& q : parts) {
            if (q.pitch == q.cols) spans.push_back({q.offset, q.rows * q.cols});
            else
                for (int64_t r = 0; r < q.rows; ++r) spans.push_back({q.offset + r * q.pitch, q.cols});
        }
        std::sort(spans.begin(), spans.end());
        std::vector<Gap> gap;
        int64_t at = 0;
        const auto between = [&](int64_t to) {
            for (; at < to; at += kGapChunk) gap.push_back({at, std::min(kGapChunk, to - at)});
        };
        for (const auto& q : spans) {
            between(q.first);
            at = q.first + q.second;
        }
        between(d);
        if ((int64_t)gap.size() > 4 * kMostTiles) {
            delete p;
            return op_error(GMC_EINVAL, me, "too many pieces outside the matrices");
        }
        p->norms = norm.size();
        p->pieces = pack.size();
        p->grams = gram.size();
        p->applies = apply.size();
        p->gaps = gap.size();
        std::vector<char> host;
        const auto add = [&](const void* from, size_t bytes) {
            const size_t here = host.size();
            host.resize(here + (bytes + 255) / 256 * 256);
            if (bytes) memcpy(host.data() + here, from, bytes);
            return here;
        };
        const size_t at_mats = add(mats.data(), mats.size() * sizeof(Mat)), at_norm = add(norm.data(), norm.size() * sizeof(Tile)),
                     at_pack = add(pack.data(), pack.size() * sizeof(Tile)), at_gram = add(gram.data(), gram.size() * sizeof(Tile)),
                     at_apply = add(apply.data(), apply.size() * sizeof(Tile)), at_gap = add(gap.data(), gap.size() * sizeof(Gap));
        if (hipGetDevice(&p->device) != hipSuccess) {
            delete p;
            return op_error(GMC_EDEVICE, me, "no current device");
        }
        if (!host.empty()) {
            const hipError_t e = hipMalloc(&p->table, host.size());
            if (e != hipSuccess) {
                (void)hipGetLastError();
                delete p;
                return op_error(GMC_ENOMEM, me, hipGetErrorString(e));
            }
            const hipError_t f = hipMemcpy(p->table, host.data(), host.size(), hipMemcpyHostToDevice);
            if (f != hipSuccess) {
                (void)hipGetLastError();
                (void)hipFree(p->table);
                delete p;
                return op_error(GMC_EDEVICE, me, hipGetErrorString(f));
            }
        }
        char* t = static_cast<char*>(p->table);
        p->mats = reinterpret_cast<const Mat*>(t + at_mats);
        p->norm = reinterpret_cast<const Tile*>(t + at_norm);
        p->pack = reinterpret_cast<const Tile*>(t + at_pack);
        p->gram = reinterpret_cast<const Tile*>(t + at_gram);
        p->apply = reinterpret_cast<const Tile*>(t + at_apply);
        p->gap = reinterpret_cast<const Gap*>(t + at_gap);
        *out = p;
        return GMC_OK;
    } catch (const std::bad_alloc&) {
        delete p;
        return op_error(GMC_ENOMEM, me, "host memory");
    } catch (...) {
        delete p;
        return op_error(GMC_EINVAL, me, "the plan could not be made");
    }
}

void gmc_matrices_destroy(gmc_matrices* plan) {
    if (!plan) return;
    if (plan->table) (void)hipFree(plan->table);
    delete plan;
}

int64_t gmc_matrices_workspace(const gmc_matrices* plan) { return plan ? layout(plan, nullptr).bytes : -1; }

gmc_status gmc_orthogonalize(void* hip_stream, const gmc_matrices* plan, int32_t dtype, const void* x_dev, void* out_dev,
                             int32_t steps, const double* coefficients, double eps, double alpha, void* workspace_dev,
                             int64_t workspace_bytes) {
    const char* me = "gmc_orthogonalize";
    const gmc_status ok = matrices_check(me, plan, dtype, steps, coefficients, eps, workspace_dev, workspace_bytes);
    if (ok != GMC_OK) return ok;
    if (!x_dev || !out_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    if (!isfinite((float)alpha)) return op_error(GMC_EINVAL, me, "alpha must be finite in fp32");
    const int64_t bytes = plan->d * type_size(dtype);
    const Span x(x_dev, bytes), out(out_dev, bytes), scratch(workspace_dev, plan->n ? gmc_matrices_workspace(plan) : 0);
    if (!apart({out, scratch}, {}) || !apart({scratch}, {x}) || (x_dev != out_dev && !apart({out}, {x})))
        return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    GMC_BY_TYPE(dtype, {
        if (plan->gaps && x_dev != out_dev)
            matrix_gaps<DT, false><<<dim3((unsigned)plan->gaps), 256, 0, st>>>(plan->gap, x_dev, nullptr, out_dev);
        if (plan->n) {
            VectorArgs v{};
            v.x = x_dev;
            ProductArgs a{};
            a.mats = plan->mats;
            a.out = out_dev;
            a.alpha = (float)alpha;
            run_steps<DT, false>(plan, layout(plan, workspace_dev), {steps, coefficients, eps}, v, a, st);
        }
    });
    return op_launched(me);
}

gmc_status gmc_orthogonal_step(void* hip_stream, const gmc_matrices* plan, int32_t dtype, const float* w_dev,
                               const void* update_dev, float* momentum_dev, float* w_out_dev, double rate, double mu,
                               int32_t nesterov, double decay, int32_t steps, const double* coefficients, double eps,
                               void* workspace_dev, int64_t workspace_bytes) {
    const char* me = "gmc_orthogonal_step";
    const gmc_status ok = matrices_check(me, plan, dtype, steps, coefficients, eps, workspace_dev, workspace_bytes);
    if (ok != GMC_OK) return ok;
    if (!w_dev || !update_dev || !w_out_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    if (!isfinite((float)rate) || !isfinite((float)decay)) return op_error(GMC_EINVAL, me, "rate and decay must be finite in fp32");
    if (!(mu >= 0.0 && mu <= 1.0)) return op_error(GMC_EINVAL, me, "mu must be in [0, 1]");
    const Span w(w_dev, plan->d * 4), update(update_dev, plan->d * type_size(dtype)), momentum(momentum_dev, plan->d * 4),
        out(w_out_dev, plan->d * 4), scratch(workspace_dev, plan->n ? gmc_matrices_workspace(plan) : 0);
    if (!apart({out, momentum, scratch}, {update}) || !apart({momentum, scratch}, {w}) || (w_dev != w_out_dev && !apart({out}, {w})))
        return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    GMC_BY_TYPE(dtype, {
        if (plan->gaps)
            matrix_gaps<DT, true><<<dim3((unsigned)plan->gaps), 256, 0, st>>>(plan->gap, update_dev, w_dev, w_out_dev);
        if (plan->n) {
            VectorArgs v{};
            v.x = update_dev;
            v.momentum = momentum_dev;
            v.mu = (float)mu;
            v.nesterov = nesterov != 0;
            ProductArgs a{};
            a.mats = plan->mats;
            a.out = w_out_dev;
            a.w = w_dev;
            a.alpha = (float)rate;
            a.keep = (float)(1.0 - decay);
            run_steps<DT, true>(plan, layout(plan, workspace_dev), {steps, coefficients, eps}, v, a, st);
        }
    });
    return op_launched(me);
}

}  // extern "C"
