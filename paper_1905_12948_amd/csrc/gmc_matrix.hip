// Orthogonalised matrices of a flat vector (gmc_orthogonalize and
// gmc_orthogonal_step in include/gmc.h): Newton-Schulz steps
//   X <- (a I + b G + c G G) X,  G = X X^T,
// from X = M / (|M| + eps), |.| the Frobenius norm, M taken on its side where it
// has more rows than columns (the steps commute with transposition): X is m x n,
// m <= n.
//
// Precision.  The steps amplify small singular values by up to prod a_k (485 for
// the five usual ones) and with them any rounding of X, so X, G and the polynomial
// are kept to 22 bits: each value as two halves, hi = f16(v) and lo = f16(2^11 (v - hi)), v the value
// times a power of two (X and G: 2^13, the polynomial: 2^10 or less).  lo has a scale of its own so that it
// reaches f16's smallest number, 2^-24, no sooner than hi does: what is lost of a value is 2^-22 of it, or 2^-49 of 1
// (the polynomial: 2^-46) where that is more.  Without it, 2^-38: rows 10^-5 the size of the others came out
// 6e-4 off in a 1000 x 1100 matrix, so 2e-6, as with products in 32 bits; rows of 10^-7 4e-5 (32 bits 2e-6).  A product is
// hi hi + 2^-11 (hi lo + lo hi) on the f16 matrix instructions, in two sums of 32 bits: what is left out, lo lo,
// is 2^-22 of it.  The result is nearer to the 64-bit one than with products in 32 bits (its error 0.4 to 0.75 of theirs).
//
// Where |M| is not far above eps X is small, as small as M, and would leave f16's range: what
// is held is Y = X / theta, theta <= 1 a number of the matrix and the step: at first
// |M| / (|M| + eps), so that |Y| = 1, then as much more as the step's polynomial can
// amplify, up to 1.  In Y a step is Y <- (theta / theta') (a I + b theta^2 G + c theta^4 G G) Y.
//
// Layout.  X's transpose, G and the polynomial are stored in the order the matrix
// instructions read: blocks of 32 rows x 16 columns, lane l's eight neighbours of row
// l % 32 as 16 bytes at l * 16, hi then lo.  X's product and G's square read every operand
// along its contraction (the polynomial and X^T along m; G is its own transpose), so a
// tile's blocks go to shared memory and to registers in whole kilobytes, with no bank
// conflict and no swizzle.  G's product, along n, turns X^T on its way from shared memory to
// registers: a copy of X along n, written by every step's last launch, costs more there (ResNet-50's
// matrices 106 us, without it 80; the server's step 1.08 ms and 0.97) than the turning does in G's
// product (2048 x 2048: 40 us, turned 41).  Rows and columns are padded with zeros to 32, which the
// steps keep.
//
// What bounds it.  Three products of halves for one in 32 bits: X's product of 4096 x 4096 at 1230 to 1270 TFLOP/s of
// them, 90 to 93 % of the 1366 a library's product of f16 matrices of that size reaches, G's and its square at 970 to 1010 of
// what their tiles compute (all hold the clock at 1.6 GHz of 2.4: power).  Many matrices of few rows are bound by what a step's last launch
// reads and writes (ResNet-50: 8 bytes a component and step, 3.5 TB/s with the loads that tiles share), small
// ones by the launches' chains (3 of 768 x 768: 12 us a launch, of which 2.5 us are the launch's and 2.5 its end's).
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

constexpr float kScaleX = 0x1p13f;                       // of X and G
constexpr float kScaleLo = 0x1p11f;                      // of a low half, beside its value's
constexpr int kSide = 64;                                // side of the pieces the vector is read in
constexpr int kParts = 1024;                             // partial sums of a matrix's squares
constexpr int64_t kGapChunk = 1024;                      // components outside the matrices, a workgroup (more in long vectors)
constexpr int kMostSteps = 64;

// A matrix of the plan.  m <= n are its sides, mb and nb their number in blocks of 32.
struct Mat {
    int64_t offset, pitch;
    int64_t x, g;      // first block of X^T and of G
    int32_t rows, cols, m, n, mb, nb;
    int32_t flip;      // rows > cols: X is the transpose
    float scale;
    int32_t part, parts;
};

// What a workgroup does: of the vector's launches `count` pieces of a matrix from (i, j) on, of a
// product's one tile (i, j), its contraction from block `first` to `last`; slot: where a part of
// a tile's sum goes, -1 for a whole tile.  A joining launch adds `count` slots from `slot` on.
struct Tile {
    int32_t mat, i, j, count;
    int32_t first, last, slot, unused;
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
    _Float16* XT;
    float* theta;              // [matrices][kMostSteps + 1]
    int32_t steps;
    float growth[kMostSteps];  // by which a step amplifies at most, 1 or more
};

// What is orthogonalised, from the update and the momentum that holds it already.
__device__ __forceinline__ float direction(const VectorArgs& a, float u, float v) { return a.nesterov ? u + a.mu * v : v; }

// Four neighbours, of which the matrix has n.
template <int DT>
__device__ __forceinline__ void load4(const typename Elem<DT>::T* p, int n, float (&f)[4]) {
    if (n >= 4) {
        if constexpr (DT == GMC_F32) {
            Vec<DT, 4>::load(p).unpack(f);
        } else {
            float a[2], b[2];
            Vec<DT, 2>::load(p).unpack(a);
            Vec<DT, 2>::load(p + 2).unpack(b);
            f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = e < n ? Elem<DT>::up(p[e]) : 0.0f;
    }
}

// Sums of squares in 64 bits (no 32-bit value's square leaves their range), and the
// momentum's update on the way.
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
        const int c = pc * kSide + c0, n = m.cols - c;   // columns from here on
        // all of a piece's loads before the first is used
        float u[4][4], w[4][4];
        const auto place = [&](int q) { return ((int64_t)pr * kSide + r0 + 16 * q) * m.pitch + c; };
        const auto have = [&](int q) { return (int64_t)pr * kSide + r0 + 16 * q < m.rows ? n : 0; };
#pragma unroll
        for (int q = 0; q < 4; ++q) load4<DT>(x + place(q), have(q), u[q]);
        if constexpr (kStep) {
            if (a.momentum) {
                float* v = a.momentum + m.offset;
#pragma unroll
                for (int q = 0; q < 4; ++q) load4<GMC_F32>(v + place(q), have(q), w[q]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[q][e] = a.mu * w[q][e] + u[q][e];
                        u[q][e] = direction(a, u[q][e], w[q][e]);
                    }
                    if (have(q) >= 4) {
                        Vec<GMC_F32, 4> o;
                        o.pack(w[q]);
                        o.store(v + place(q));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < have(q)) v[place(q) + e] = w[q][e];
                    }
                }
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fma((double)u[q][e], (double)u[q][e], sum);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.part[m.part + t.j] = lds[0] + lds[1] + lds[2] + lds[3];
}

// Values as their two halves, two at a time (two values are converted in one operation, and what
// hi leaves, times kScaleLo, is one of the mixed-precision ones).
template <int N, class H>
__device__ __forceinline__ void split(const float (&v)[N], H& hi, H& lo) {
    float minus = -kScaleLo;   // not known to be: what hi leaves would be a conversion, a product and a difference
    asm("" : "+s"(minus));
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        f32x2 x;
        x.x = v[e];
        x.y = v[e + 1];
        const f16x2 h = __builtin_convertvector(x, f16x2);
        f32x2 r;
        r.x = __builtin_fmaf((float)h.x, minus, v[e] * kScaleLo);
        r.y = __builtin_fmaf((float)h.y, minus, v[e + 1] * kScaleLo);
        const f16x2 l = __builtin_convertvector(r, f16x2);
        hi[e] = h.x;
        hi[e + 1] = h.y;
        lo[e] = l.x;
        lo[e + 1] = l.y;
    }
}

// What a wavefront's lanes have written to shared memory before is there for what they read after.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// theta of the steps (see above); NaN stays.
__device__ __forceinline__ float first_theta(double norm, double eps) { return norm == 0.0 ? 1.0f : (float)(norm / (norm + eps)); }
__device__ __forceinline__ float next_theta(float theta, float growth) { return fminf(theta * growth, 1.0f) + 0.0f * theta; }

// The transpose of X, the matrix over its norm, in halves.
template <int DT, bool kStep>
__global__ __launch_bounds__(256) void matrix_pack(VectorArgs a) {
    typedef typename Elem<DT>::T T;
    __shared__ float in[kSide][kSide + 1];
    __shared__ double lds[4];
    const Tile t = a.tiles[blockIdx.x];
    const Mat m = a.mats[t.mat];
    const T* x = static_cast<const T*>(a.x) + m.offset;
    // piece (i, j) of X is piece (j, i) of a matrix on its side
    const int pr = m.flip ? t.j : t.i, pc = m.flip ? t.i : t.j;
    const int c0 = threadIdx.x & 63, r0 = threadIdx.x >> 6, c = pc * kSide + c0;
    const bool there = c < m.cols;
    float u[16], v[16];
    // past the last row and column those are read again, and not used
    const auto at = [&](int q) {
        const int64_t r = (int64_t)pr * kSide + r0 + 4 * q;
        return (r < m.rows ? r : (int64_t)m.rows - 1) * m.pitch + (there ? c : m.cols - 1);
    };
#pragma unroll
    for (int q = 0; q < 16; ++q) u[q] = Elem<DT>::up(x[at(q)]);
    if constexpr (kStep) {
        if (a.momentum) {
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = a.momentum[m.offset + at(q)];
        }
    }
    double sum = 0.0;
    for (int k = threadIdx.x; k < m.parts; k += 256) sum += a.part[m.part + k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        if constexpr (kStep)
            if (a.momentum) u[q] = direction(a, u[q], v[q]);
        in[r0 + 4 * q][c0] = there && (int64_t)pr * kSide + r0 + 4 * q < m.rows ? u[q] : 0.0f;
    }
    __syncthreads();
    const double norm = sqrt(lds[0] + lds[1] + lds[2] + lds[3]);
    const double inv = norm == 0.0 ? 0.0 : (double)kScaleX / norm;
    if (t.i == 0 && t.j == 0 && threadIdx.x == 0) {
        float v = first_theta(norm, a.eps);
        float* theta = a.theta + t.mat * (kMostSteps + 1);
        theta[0] = v;
        for (int k = 0; k < a.steps; ++k) theta[k + 1] = v = next_theta(v, a.growth[k]);
    }
    const int64_t km = 2 * (int64_t)m.mb;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        // eight neighbours of a column of X
        const int unit = threadIdx.x + 256 * u, j = unit & 63, k8 = unit >> 6;
        f16x8 hi, lo;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = 8 * k8 + e;
            f[e] = (float)((double)(m.flip ? in[j][i] : in[i][j]) * inv);
        }
        split(f, hi, lo);
        const int rb = t.j * 2 + (j >> 5), kb = t.i * 4 + (k8 >> 1);
        if (rb < m.nb && kb < km) {
            _Float16* o = a.XT + (m.x + rb * km + kb) * 1024 + ((j & 31) + 32 * (k8 & 1)) * 8;
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
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < g.len; i += 256) {
        if constexpr (kStep) static_cast<float*>(out)[g.at + i] = w[g.at + i] + Elem<DT>::up(x[i]);
        else static_cast<T*>(out)[g.at + i] = x[i];
    }
}

// (1 - decay) w + step as keep w - decay w + step, the small terms first: 1 - decay in 32 bits is off by up to
// 2^-25, the same way in every step, and a decay below that would be none.
__device__ __forceinline__ float decayed(float w, float keep, float decay, float step) {
    return __builtin_fmaf(keep, w, fabsf(w) < INFINITY ? __builtin_fmaf(-decay, w, step) : step);
}

// -- products ---------------------------------------------------------------------

enum { kGram, kPoly, kApply, kLast, kLastStep };

struct ProductArgs {
    const Mat* mats;
    const Tile* tiles;
    const _Float16 *XT, *G, *B;  // what the mode reads
    _Float16 *XTo, *Go, *Bo;     // and writes
    const float* theta;  // this step's of the first matrix
    float a, b, c, scale;   // of the step, and what the polynomial is held times
    float* slots;        // parts of tiles' sums
    void* out;           // kLast, kLastStep
    const float* w;      // kLastStep
    float alpha, keep, decay;
};

// The rows and columns of a mode's tiles, in blocks; i and j where a matrix on its side is written last.
template <int kMode>
struct Sides {
    static constexpr bool kEnd = kMode == kLast || kMode == kLastStep, kEven = kMode == kGram || kMode == kPoly;
    bool flip;
    int i, j, rows, cols;
    __device__ __forceinline__ Sides(const Mat& m, const Tile& t) {
        flip = kEnd && m.flip;
        i = flip ? t.j : t.i;
        j = flip ? t.i : t.j;
        rows = !kEven && flip ? m.nb : m.mb;
        cols = kEven || flip ? m.mb : m.nb;
    }
};

// What the mode makes of a wavefront's blocks of D, from (ib, jb) on.  turn: 32 x 33 words of shared memory
// of the wavefront's own.  Of a block lane l has column l % 32, rows 8 g + 4 (l / 32) + e in
// entry 4 g + e.
template <int kWide, int kMode, int DT>
__device__ __forceinline__ void finish_blocks(const ProductArgs& a, const Mat& m, const Tile& t, const Sides<kMode>& sides, int ib0,
                                              int jb0, const f32x16 (&acc)[kWide][kWide], float* turn) {
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const float theta = kMode == kGram ? 1.0f : a.theta[t.mat * (kMostSteps + 1)];
    // the last step takes X's scale off here: theta may be so small that what it is multiplied with would lose bits by it
    const float ratio = kMode == kApply ? theta / a.theta[t.mat * (kMostSteps + 1) + 1] : 1.0f / kScaleX;
    // d <- v d, of the polynomial a I + u hi + ul lo + v d
    const float u = a.b * (theta * theta) * (a.scale / kScaleX), ul = u * (1.0f / kScaleLo);
    const float v = kMode == kPoly ? a.c * (theta * theta) * (theta * theta) * (a.scale / kScaleX / kScaleX) : ratio / a.scale;
    const auto inside = [&](int i, int j) { return ib0 + i < sides.rows && jb0 + j < sides.cols; };
    // entry (i, j) where its row is j: block (jb, 2 ib + g / 2), lane col + 32 (g % 2), halves 4 half + e
    const auto spot = [&](int i, int j) { return ((int64_t)(jb0 + j) * 2 * sides.rows + 2 * (ib0 + i)) * 1024 + col * 8 + 4 * half; };
    // in the vector
    const auto row = [](int e) { return 8 * (e >> 2) + (e & 3); };
    const auto known = [&](int i, int j, int e) {
        return ((ib0 + i + 1) * 32 <= m.rows || (ib0 + i) * 32 + 4 * half + row(e) < m.rows) &&
               ((jb0 + j + 1) * 32 <= m.cols || (jb0 + j) * 32 + col < m.cols);
    };
    const auto where = [&](int i, int j) {
        return m.offset + (int64_t)((ib0 + i) * 32 + 4 * half) * m.pitch + (jb0 + j) * 32 + col;
    };
    // all that is read before anything is written: a wait for each block's would follow the other's stores
    constexpr bool kAdds = kMode == kPoly, kParts = kMode == kLastStep;
    f16x4 hi[kAdds ? kWide : 1][kAdds ? kWide : 1][4], lo[kAdds ? kWide : 1][kAdds ? kWide : 1][4];
    float w[kParts ? kWide : 1][kParts ? kWide : 1][16];
    if constexpr (kAdds || kParts) {
        const _Float16* add = a.G + m.g * 1024;
#pragma unroll
        for (int i = 0; i < kWide; ++i)
#pragma unroll
            for (int j = 0; j < kWide; ++j)
                if (inside(i, j)) {
                    if constexpr (kAdds) {
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            hi[i][j][g] = *reinterpret_cast<const f16x4*>(add + spot(i, j) + (g >> 1) * 1024 + (g & 1) * 256);
                            lo[i][j][g] = *reinterpret_cast<const f16x4*>(add + spot(i, j) + (g >> 1) * 1024 + (g & 1) * 256 + 512);
                        }
                    }
                    if constexpr (kParts) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[i][j][e] = known(i, j, e) ? a.w[where(i, j) + row(e) * m.pitch] : 0.0f;
                    }
                }
    }
#pragma unroll
    for (int i = 0; i < kWide; ++i)
#pragma unroll
        for (int j = 0; j < kWide; ++j) {
            if (!inside(i, j)) continue;
            const int ib = ib0 + i, jb = jb0 + j;
            const int64_t place = spot(i, j);
            f32x16 d = acc[i][j];
            if constexpr (kMode == kPoly) {
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        d[4 * g + e] = __builtin_fmaf((float)hi[i][j][g][e], u, __builtin_fmaf((float)lo[i][j][g][e], ul, v * d[4 * g + e]));
                if (ib == jb) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) d[e] += row(e) + 4 * half == col ? a.a * a.scale : 0.0f;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) d[e] *= kMode == kGram ? 1.0f / kScaleX : v;
            }
            if constexpr (kMode == kLast || kMode == kLastStep) {
                typedef typename Elem<DT>::T T;
                const float factor = a.alpha * m.scale * theta;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (known(i, j, e)) {
                        const int64_t at = where(i, j) + row(e) * m.pitch;
                        if constexpr (kMode == kLastStep) static_cast<float*>(a.out)[at] = decayed(w[i][j][e], a.keep, a.decay, factor * d[e]);
                        else static_cast<T*>(a.out)[at] = Elem<DT>::down(factor * d[e]);
                    }
                continue;
            }
            _Float16* o = (kMode == kGram ? a.Go + m.g * 1024 : kMode == kPoly ? a.Bo + m.g * 1024 : a.XTo + m.x * 1024) + place;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f16x4 hi, lo;
                float f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = d[4 * g + e];
                split(f, hi, lo);
                *reinterpret_cast<f16x4*>(o + (g >> 1) * 1024 + (g & 1) * 256) = hi;
                *reinterpret_cast<f16x4*>(o + (g >> 1) * 1024 + (g & 1) * 256 + 512) = lo;
            }
            if (kMode == kApply || t.i == t.j) continue;
            // and where its row is i, by way of shared memory
#pragma unroll
            for (int e = 0; e < 16; ++e) turn[(8 * (e >> 2) + 4 * half + (e & 3)) * 33 + col] = d[e];
            wave_order();
            o = (kMode == kGram ? a.Go + m.g * 1024 : a.Bo + m.g * 1024) + ((int64_t)ib * 2 * sides.cols + 2 * jb) * 1024 + lane * 8;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                f16x8 hi, lo;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = turn[col * 33 + 16 * k + 8 * half + e];
                split(f, hi, lo);
                *reinterpret_cast<f16x8*>(o + k * 1024) = hi;
                *reinterpret_cast<f16x8*>(o + k * 1024 + 512) = lo;
            }
            wave_order();
        }
}

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

// Four neighbours of each of 16 lanes, turned: lane l of them gets entry l % 4 of lanes l / 4, l / 4 + 4, + 8 and + 12.
__device__ __forceinline__ f16x4 turned(const _Float16* p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(f16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}

// The first of a lane's vectors of a slot.
template <int kWide>
__device__ __forceinline__ int64_t slot_of(int slot, int wave, int lane) {
    return ((int64_t)slot * 4 + wave) * (kWide * kWide * 4 * 64) + lane;
}

// One tile of D = P Q^T, both along their contraction, by four wavefronts of kWide x
// kWide blocks each, and what the mode makes of it:
//   kGram   P = Q = X            G = D, X read as X^T
//   kPoly   P = Q = G            B = a I + b G + c D
//   kApply  P = B, Q = X^T       X^T <- D^T
//   kLast   the same, or P = X^T and Q = B for a matrix on its side, into the vector
// or, of a tile whose contraction is cut, its part of the sum for matrix_join.  G and B are symmetric: tiles with j <= i, written to both places.
template <int kWide, int kStages, int kMode, int DT>
__global__ __launch_bounds__(256, kStages == 4 ? 2 : 3) void matrix_product(ProductArgs a) {
    constexpr int kBlocks = 2 * kWide;                 // of 32 rows, on each side of the tile
    constexpr int kDeep = kWide == 2 ? 1 : 2;          // 16 columns, of a stage
    constexpr int kChunks = 2 * kBlocks * kDeep * 2;   // kilobytes of a stage: sides, blocks, columns, halves
    // arrays of their own, so that a wait for one stage's loads is none for the others'
    __shared__ _Float16 stage0[kChunks * 512], stage1[kChunks * 512], stage2[kChunks * 512], stage3[kStages == 4 ? kChunks * 512 : 8];
    const Tile t = a.tiles[blockIdx.x];
    if (t.mat < 0) return;   // fills an XCD's list
    const Mat m = a.mats[t.mat];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const Sides<kMode> sides(m, t);
    const _Float16* P = (kMode == kPoly ? a.G + m.g * 1024 : kMode == kGram || sides.flip ? a.XT + m.x * 1024 : a.B + m.g * 1024);
    const _Float16* Q = (kMode == kPoly ? a.G + m.g * 1024 : kMode == kGram || !sides.flip ? a.XT + m.x * 1024 : a.B + m.g * 1024);
    const int64_t row = (int64_t)m.mb * 2048;   // halves of a row of blocks

    // chunk c of a stage: side, block, 16 columns, half; a wavefront takes every fourth.
    // Blocks beyond the matrix are read as its last one and not written.
    const _Float16* from[kChunks / 4];
#pragma unroll
    for (int k = 0; k < kChunks / 4; ++k) {
        const int c = k * 4 + wave, side = c / (kChunks / 2), b = c / (2 * kDeep) % kBlocks;
        int rb = (side ? sides.j : sides.i) * kBlocks + b;
        const int most = (side ? sides.cols : sides.rows) - 1;
        rb = rb < most ? rb : most;
        from[k] = kMode == kGram ? P + t.first * row + (int64_t)rb * 2048 + (c & 1) * 512 + c % (2 * kDeep) / 2 * 128
                                 : (side ? Q : P) + rb * row + (int64_t)t.first * 2048 + (c % (2 * kDeep)) * 512;
    }
    // A lane's part.  G's product reads of 16 rows of X^T (of a row of blocks the k-th sixteen, or the stage's) 32 columns: lane l
    // brings eight neighbours, the l / 16-th of a row, so that 16 lanes read 256 bytes; their rows are
    // exchanged by fours so that what turns them meets all banks.
    const unsigned part = kMode != kGram ? lane * 8 : (lane >> 5) * 1024 + ((lane >> 4) & 1) * 256 + ((lane & 15) ^ (4 * (lane >> 4))) * 8;
    f32x16 acc[kWide][kWide], cross[kWide][kWide];   // hi hi; hi lo + lo hi, times kScaleLo
#pragma unroll
    for (int i = 0; i < kWide; ++i)
#pragma unroll
        for (int j = 0; j < kWide; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = cross[i][j][e] = 0.0f;
    const int wi = (wave >> 1) * kWide, wj = (wave & 1) * kWide;   // the wavefront's first blocks
    const int stages = (t.last - t.first) * 2 / kDeep;
    const auto fetch = [&](int s, int k, _Float16* to) {
        s = s < stages ? s : stages - 1;   // the count of loads under way stays what the waits take it for
        const int64_t at = kMode != kGram ? (int64_t)s * (kDeep * 1024) : kDeep == 2 ? s * row : (s >> 1) * row + (s & 1) * 128;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from[k] + at + part),
                                         (__attribute__((address_space(3))) void*)(to + (k * 4 + wave) * 512), 16, 0, 0);
    };
    // A wavefront's operands of a stage: of each 16 columns kWide blocks of P in their halves, then of Q.
    constexpr int kReads = kDeep * 4 * kWide, kProducts = kDeep * 3 * kWide * kWide, kLoads = kChunks / 4;
    // (of G's product: lane l reads four neighbours of row 8 (l / 32) + l / 4 % 4, and then of the fourth after it, of
    // columns 16 (l / 16 % 2) + 4 (l % 4), and gets four rows' of column l % 32)
    const int eighth = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    const int turn_from = 128 * eighth + (((lane >> 2) & 3) + ((8 * (lane >> 5)) ^ (4 * eighth))) * 8 + 4 * (lane & 1);
    const auto read = [&](f16x8 (&o)[kReads], int r, const _Float16* here) {
        const int k = r / (4 * kWide), q = r / (2 * kWide) % 2, i = r / 2 % kWide, h = r % 2;
        const _Float16* chunk = here + (((q ? kBlocks + wj + i : wi + i) * kDeep + k) * 2 + h) * 512;
        if constexpr (kMode == kGram) {
            const f16x4 one = turned(chunk + turn_from), two = turned(chunk + (turn_from ^ 32));
            o[r] = __builtin_shufflevector(one, two, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            o[r] = reinterpret_cast<const f16x8*>(chunk)[lane];
        }
    };
    // Stage s + 1 is in shared memory and stage s has been read by all, whose place the loads of
    // stage s + kStages take; those of the stages between stay under way.  The operands of s + 1 are read
    // and the loads issued between the products of s, one after each: in front of them they
    // hold the products up (2048 x 2048, one workgroup a CU: X's product 59 us, so 53; with what else followed 48).
    const auto step = [&](int s, const f16x8 (&now)[kReads], f16x8 (&then)[kReads], const _Float16* after, _Float16* here) {
        wait_stage<(kStages - 2) * kLoads>();
#pragma unroll
        for (int n = 0; n < kProducts; ++n) {
            const int k = n / (3 * kWide * kWide), part = n / (kWide * kWide) % 3, i = n / kWide % kWide, j = n % kWide;
            f32x16& sum = part ? cross[i][j] : acc[i][j];
            sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[k * 4 * kWide + 2 * i + (part == 2)],
                                                         now[k * 4 * kWide + 2 * kWide + 2 * j + (part == 1)], sum, 0, 0, 0);
#pragma unroll
            for (int r = n * (kReads + kLoads) / kProducts; r < (n + 1) * (kReads + kLoads) / kProducts; ++r) {
                if (r < kReads) read(then, r, after);
                else fetch(s + kStages, r - kReads, here);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    f16x8 one[kReads], two[kReads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) fetch(0, k, stage0);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) fetch(1, k, stage1);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) fetch(2, k, stage2);
    if constexpr (kStages == 4) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) fetch(3, k, stage3);
    }
    wait_stage<(kStages - 1) * kLoads>();
#pragma unroll
    for (int r = 0; r < kReads; ++r) read(one, r, stage0);
    int s = 0;
    if constexpr (kStages == 4) {
        for (; s + 4 <= stages; s += 4) {
            step(s, one, two, stage1, stage0);
            step(s + 1, two, one, stage2, stage1);
            step(s + 2, one, two, stage3, stage2);
            step(s + 3, two, one, stage0, stage3);
        }
        if (s < stages) step(s, one, two, stage1, stage0);
        if (s + 1 < stages) step(s + 1, two, one, stage2, stage1);
        if (s + 2 < stages) step(s + 2, one, two, stage3, stage2);
    } else {
        for (; s + 6 <= stages; s += 6) {
            step(s, one, two, stage1, stage0);
            step(s + 1, two, one, stage2, stage1);
            step(s + 2, one, two, stage0, stage2);
            step(s + 3, two, one, stage1, stage0);
            step(s + 4, one, two, stage2, stage1);
            step(s + 5, two, one, stage0, stage2);
        }
        if (s < stages) step(s, one, two, stage1, stage0);
        if (s + 1 < stages) step(s + 1, two, one, stage2, stage1);
        if (s + 2 < stages) step(s + 2, one, two, stage0, stage2);
        if (s + 3 < stages) step(s + 3, two, one, stage1, stage0);
        if (s + 4 < stages) step(s + 4, one, two, stage2, stage1);
    }
    wait_stage<0>();   // no load is under way and shared memory is free
#pragma unroll
    for (int i = 0; i < kWide; ++i)
#pragma unroll
        for (int j = 0; j < kWide; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = __builtin_fmaf(cross[i][j][e], 1.0f / kScaleLo, acc[i][j][e]);

    static_assert(2 * 32 * 33 * 4 <= kChunks * 1024, "two wavefronts' blocks fit a stage");
    float* turn = reinterpret_cast<float*>(wave < 2 ? stage0 : stage1) + (wave & 1) * 32 * 33;
    if (t.slot >= 0) {
        f32x4* o = reinterpret_cast<f32x4*>(a.slots) + slot_of<kWide>(t.slot, wave, lane);
#pragma unroll
        for (int i = 0; i < kWide; ++i)
#pragma unroll
            for (int j = 0; j < kWide; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * g + e];
                    o[((i * kWide + j) * 4 + g) * 64] = v;
                }
        return;
    }
    finish_blocks<kWide, kMode, DT>(a, m, t, sides, sides.i * kBlocks + wi, sides.j * kBlocks + wj, acc, turn);
}

// The tiles whose contraction was cut: their parts added in order, a wavefront a block.
template <int kWide, int kMode>
__global__ __launch_bounds__(256) void matrix_join(ProductArgs a) {
    __shared__ float turn[4][32 * 33];
    const Tile t = a.tiles[blockIdx.x / (kWide * kWide)];
    const Mat m = a.mats[t.mat];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int block = blockIdx.x % (kWide * kWide), i = block / kWide, j = block % kWide;   // of each wavefront's
    f32x16 acc[1][1];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][0][e] = 0.0f;
    constexpr int64_t kSlot = kWide * kWide * 4 * 4 * 64;
    const f32x4* p = reinterpret_cast<const f32x4*>(a.slots) + slot_of<kWide>(t.slot, wave, lane) + block * 4 * 64;
#pragma unroll 4
    for (int k = 0; k < t.count; ++k) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 v = p[k * kSlot + g * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[0][0][4 * g + e] += v[e];
        }
    }
    const Sides<kMode> sides(m, t);
    finish_blocks<1, kMode, GMC_F32>(a, m, t, sides, (sides.i * 2 + (wave >> 1)) * kWide + i, (sides.j * 2 + (wave & 1)) * kWide + j, acc,
                                     turn[wave]);
}

// -- small matrices -----------------------------------------------------------------

struct SmallArgs {
    VectorArgs in;
    float c[kMostSteps][4];
    void* out;
    const float* w;
    float alpha, keep, decay;
};

constexpr int kSmallThreads = 1024, kSmallBlocks = 40;   // 4 KB each of 160 KB: X^T and G of 32 x 32 blocks
constexpr int kSmallSide = 4;                            // the most blocks of the shorter side

// Matrices of which X^T and G fit the shared memory of one CU: all steps in one launch, a workgroup a
// matrix, a wavefront every sixteenth block of what a phase computes.  The polynomial takes G's place, and
// X^T its own, once all have read them.  G's product turns X^T as above; rows of X^T are exchanged by
// fours within 16 so that this meets all banks.  What shared memory is left takes the parts
// of G that wavefronts without a block of their own sum, and then the polynomial.  It is bound by that
// chain, about 4 us a step: 64 x 147 in five steps 31 us (by the launches above 58), 64 x 576 64 (73), 128 x 192 60
// (67); 600 of 128 x 192, three a CU one after the other, 205 to 243 (444).
template <int DT, bool kStep, int mb>
__global__ __launch_bounds__(kSmallThreads) void matrix_small(SmallArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int kWaves = kSmallThreads / 64, kMost = (kSmallBlocks - mb * mb) / mb * mb;   // blocks of X
    constexpr int kOwn = (kMost + kWaves - 1) / kWaves, kUnits = (kMost * 128 + kSmallThreads - 1) / kSmallThreads;
    __shared__ f16x8 lds[kSmallBlocks * 256];
    const Mat m = a.in.mats[blockIdx.x];
    int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int nb = m.nb;   // mb = m.mb
    // a block of 32 rows and 32 columns is four times 64 vectors: 16 columns' hi and lo, twice
    f16x8 *XT = lds, *G = XT + mb * nb * 256;
    double* sums = reinterpret_cast<double*>(G);
    // X in 32 bits, where X^T is later: [i][j], four neighbours exchanged with others by the row so that a
    // column's walk and a row's both meet all banks
    float* raw = reinterpret_cast<float*>(XT);
    const auto spot = [&](int i, int j) { return i * 32 * nb + (j ^ (i & 7) << 2); };
    const int units = 32 * mb * 32 * nb;
    {
        const T* x = static_cast<const T*>(a.in.x) + m.offset;
        float* past = kStep && a.in.momentum ? a.in.momentum + m.offset : nullptr;
        // along the matrix's own rows, padded as X is
        const int wide = 32 * (m.flip ? mb : nb);
        double sum = 0.0;
        for (int k0 = threadIdx.x; k0 < units; k0 += 8 * kSmallThreads) {
            int64_t at[8];
            float u[8], v[8];
            int r[8], c[8];
            // all loads before the first is used; outside the matrix that of its last row or column
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int k = k0 + q * kSmallThreads < units ? k0 + q * kSmallThreads : units - 1;
                r[q] = k / wide;
                c[q] = k - r[q] * wide;
                at[q] = (int64_t)(r[q] < m.rows ? r[q] : m.rows - 1) * m.pitch + (c[q] < m.cols ? c[q] : m.cols - 1);
                u[q] = Elem<DT>::up(x[at[q]]);
            }
            if (past) {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = past[at[q]];
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const bool real = r[q] < m.rows && c[q] < m.cols && k0 + q * kSmallThreads < units;
                if (past) {
                    v[q] = a.in.mu * v[q] + u[q];
                    u[q] = direction(a.in, u[q], v[q]);
                    // (a lane that reads this place for another one outside the matrix does not use it)
                    if (real) past[at[q]] = v[q];
                }
                if (!real) u[q] = 0.0f;
                sum = fma((double)u[q], (double)u[q], sum);
                if (k0 + q * kSmallThreads < units) raw[m.flip ? spot(c[q], r[q]) : spot(r[q], c[q])] = u[q];
            }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) sums[wave] = sum;
    }
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += sums[w];
    const double norm = sqrt(sum), inv = norm == 0.0 ? 0.0 : (double)kScaleX / norm;
    float theta = first_theta(norm, a.in.eps);
    {
        // eight neighbours of a column of X at a time, written when all have read theirs
        f16x8 hi[kUnits], lo[kUnits];
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            const int k = threadIdx.x + n * kSmallThreads;
            if (k >= mb * nb * 128) break;
            const int l = k & 63, b = (k >> 6) / (2 * mb), row = b * 32 + (l & 31), k0 = ((k >> 6) - b * 2 * mb) * 16 + (l >> 5) * 8;
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = (float)((double)raw[spot(k0 + e, row)] * inv);
            split(f, hi[n], lo[n]);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            const int k = threadIdx.x + n * kSmallThreads;
            if (k >= mb * nb * 128) break;
            const int at = (k >> 6) * 128 + ((k & 63) ^ (8 * ((k >> 6) & 1) + 4 * ((k >> 5) & 1)));
            XT[at] = hi[n];
            XT[at + 64] = lo[n];
        }
    }
    __syncthreads();
    // Columns 16 k of a block of P Q^T: hi hi, and hi lo + lo hi times kScaleLo
    const auto multiply = [&](f16x8 ph, f16x8 pl, f16x8 qh, f16x8 ql, f32x16& one, f32x16& two) {
        one = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, one, 0, 0, 0);
        two = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, two, 0, 0, 0);
        two = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, two, 0, 0, 0);
    };
    // Eight neighbours of rows 16 k of a block of columns of X^T, turned (see matrix_product's)
    const auto turn = [&](int b, int k, int h) {
        const int eighth = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        const int from = ((eighth >> 1) * 128 + (eighth & 1) * 32 + ((lane >> 2) & 3) + ((8 * (lane >> 5)) ^ (4 * eighth))) * 8 + 4 * (lane & 1);
        const _Float16* chunk = reinterpret_cast<const _Float16*>(XT) + ((k >> 1) * mb + b) * 2048 + (k & 1) * 128 + h * 512;
        return __builtin_shufflevector(turned(chunk + from), turned(chunk + (from ^ 32)), 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // Block ib of the polynomial's rows times block jb of X^T's rows, or (turned) the other way round
    const auto product = [&](const f16x8* B, int ib, int jb, bool turned) {
        f32x16 one, two;
#pragma unroll
        for (int e = 0; e < 16; ++e) one[e] = two[e] = 0.0f;
        const auto b = [&](int k) { return B + (ib * 2 * mb + k) * 128 + lane; };
        const auto x = [&](int k) { return XT + (jb * 2 * mb + k) * 128 + (lane ^ (8 * (k & 1) + 4 * (lane >> 5))); };
        if constexpr (kOwn <= 2) {
#pragma unroll
            for (int k = 0; k < 2 * mb; ++k) {
                if (turned) multiply(x(k)[0], x(k)[64], b(k)[0], b(k)[64], one, two);
                else multiply(b(k)[0], b(k)[64], x(k)[0], x(k)[64], one, two);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) one[e] = __builtin_fmaf(two[e], 1.0f / kScaleLo, one[e]);
        } else {
            // in one sum, the low halves' first, where a wavefront has three blocks: registers
#pragma unroll
            for (int k = 0; k < 2 * mb; ++k) {
                const f16x8 *p = turned ? x(k) : b(k), *q = turned ? b(k) : x(k);
                one = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[0], q[64], one, 0, 0, 0);
                one = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[64], q[0], one, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) one[e] *= 1.0f / kScaleLo;
#pragma unroll
            for (int k = 0; k < 2 * mb; ++k) {
                const f16x8 *p = turned ? x(k) : b(k), *q = turned ? b(k) : x(k);
                one = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[0], q[0], one, 0, 0, 0);
            }
        }
        return one;
    };
    // blocks of 4 KB that are left, and so how many wavefronts share a block of G
    const int spare = kSmallBlocks - mb * nb - mb * mb;
    f16x8* left = G + mb * mb * 256;
    int shares = kWaves / (mb * mb) < 1 + spare / (mb * mb) ? kWaves / (mb * mb) : 1 + spare / (mb * mb);
    if (shares > nb) shares = nb;
    f16x8* B = spare >= mb * mb ? left : G;
    // Entries 4 g to 4 g + 3 of block (ib, jb) where their row is j, of G and the polynomial or of X^T
    const auto half4 = [&](f16x8* base, int ib, int jb, int g, int h, int exchange) {
        return reinterpret_cast<f16x4*>(base + (jb * 2 * mb + 2 * ib + (g >> 1)) * 128 + h * 64 + ((lane & 31) ^ exchange) + 32 * (g & 1)) +
               (lane >> 5);
    };
    const auto keep4 = [&](f16x8* base, int ib, int jb, const f32x16& d, bool exchange) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f16x4 hi, lo;
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = d[4 * g + e];
            split(f, hi, lo);
            *half4(base, ib, jb, g, 0, exchange ? 4 * g : 0) = hi;
            *half4(base, ib, jb, g, 1, exchange ? 4 * g : 0) = lo;
        }
    };
    for (int step = 0; step < a.in.steps; ++step) {
        // places of blocks are worked out where they are needed: kept over the steps they would take all registers
        asm volatile("" : "+v"(lane), "+s"(wave));
        const float ca = a.c[step][0], cb = a.c[step][1], cc = a.c[step][2], scale = a.c[step][3];
        const float theta2 = theta * theta;
        f32x16 d[kOwn];
        {
            const int share = wave / (mb * mb), b = wave - share * mb * mb, ib = b / mb, jb = b - ib * mb;
            f32x16 one, two;
#pragma unroll
            for (int e = 0; e < 16; ++e) one[e] = two[e] = 0.0f;
            if (share < shares) {
                const int end = 2 * nb * (share + 1) / shares;
                for (int k = 2 * nb * share / shares; k < end; ++k) multiply(turn(ib, k, 0), turn(ib, k, 1), turn(jb, k, 0), turn(jb, k, 1), one, two);
#pragma unroll
                for (int e = 0; e < 16; ++e) one[e] = __builtin_fmaf(two[e], 1.0f / kScaleLo, one[e]);
                if (share > 0)
#pragma unroll
                    for (int e = 0; e < 16; ++e) reinterpret_cast<float*>(left)[((share - 1) * mb * mb + b) * 1024 + e * 64 + lane] = one[e];
            }
            __syncthreads();
            if (share == 0) {
                for (int k = 0; k < shares - 1; ++k)
#pragma unroll
                    for (int e = 0; e < 16; ++e) one[e] += reinterpret_cast<const float*>(left)[(k * mb * mb + b) * 1024 + e * 64 + lane];
#pragma unroll
                for (int e = 0; e < 16; ++e) one[e] *= 1.0f / kScaleX;
                keep4(G, ib, jb, one, false);
            }
        }
        __syncthreads();
        if (wave < mb * mb) {
            const int ib = wave / mb, jb = wave - ib * mb;
            f32x16 two;
#pragma unroll
            for (int e = 0; e < 16; ++e) d[0][e] = two[e] = 0.0f;
#pragma unroll
            for (int k = 0; k < 2 * mb; ++k) {
                const f16x8 *p = G + (ib * 2 * mb + k) * 128 + lane, *q = G + (jb * 2 * mb + k) * 128 + lane;
                multiply(p[0], p[64], q[0], q[64], d[0], two);
            }
            const float u = cb * theta2 * (scale / kScaleX), ul = u * (1.0f / kScaleLo), v = cc * theta2 * theta2 * (scale / kScaleX / kScaleX);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f16x4 hi = *half4(G, ib, jb, g, 0, 0), lo = *half4(G, ib, jb, g, 1, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    d[0][4 * g + e] = __builtin_fmaf((float)hi[e], u, __builtin_fmaf((float)lo[e], ul,
                                                     v * __builtin_fmaf(two[4 * g + e], 1.0f / kScaleLo, d[0][4 * g + e])));
            }
            if (ib == jb) {
#pragma unroll
                for (int e = 0; e < 16; ++e) d[0][e] += 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3) == (lane & 31) ? ca * scale : 0.0f;
            }
        }
        if (B == G) __syncthreads();
        if (wave < mb * mb) keep4(B, wave / mb, wave % mb, d[0], false);
        __syncthreads();
        const bool last = step + 1 == a.in.steps;
        const float next = last ? 0.0f : next_theta(theta, a.in.growth[step]);
        const float ratio = last ? 1.0f / kScaleX : theta / next;
        // blocks of X, whose entries have their row j in X^T; in the last step as the matrix lies
        const bool turned = last && m.flip;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const int b = wave + k * kWaves;
            if (b >= mb * nb) break;
            d[k] = product(B, b % mb, b / mb, turned);
#pragma unroll
            for (int e = 0; e < 16; ++e) d[k][e] *= ratio / scale;
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" : "+v"(lane), "+s"(wave));
        }
        if (last) {
            const float factor = a.alpha * m.scale * theta;
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                const int b = wave + k * kWaves, ib = m.flip ? b / mb : b % mb, jb = m.flip ? b % mb : b / mb;
                if (b >= mb * nb) break;
                const int r0 = ib * 32 + 4 * (lane >> 5), c = jb * 32 + (lane & 31);
                const int64_t at = m.offset + (int64_t)r0 * m.pitch + c;
                float w[16];
                if constexpr (kStep) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int r = 8 * (e >> 2) + (e & 3);
                        w[e] = r0 + r < m.rows && c < m.cols ? a.w[at + r * m.pitch] : 0.0f;
                    }
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = 8 * (e >> 2) + (e & 3);
                    if (r0 + r >= m.rows || c >= m.cols) continue;
                    if constexpr (kStep) static_cast<float*>(a.out)[at + r * m.pitch] = decayed(w[e], a.keep, a.decay, factor * d[k][e]);
                    else static_cast<T*>(a.out)[at + r * m.pitch] = Elem<DT>::down(factor * d[k][e]);
                }
            }
            return;
        }
        theta = next;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const int b = wave + k * kWaves;
            if (b >= mb * nb) break;
            keep4(XT, b % mb, b / mb, d[k], true);
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" : "+v"(lane), "+s"(wave));
        }
        __syncthreads();
    }
}

}  // namespace

}  // namespace gmc

using namespace gmc;

// The plan: the matrices, and which tile of which matrix each workgroup of a launch takes.
struct gmc_matrices {
    int64_t d = 0;
    int device = 0;
    int wide = 1, gram_wide = 1, poly_wide = 1;   // blocks a wavefront's side of a tile
    int32_t n = 0;
    int64_t blocks_x = 0, blocks_g = 0, parts = 0;
    int small = 0;             // every matrix is one workgroup's: their shorter sides' blocks
    int64_t slots = 0;         // of parts of tiles' sums, of one block a wavefront
    void* table = nullptr;     // device memory: all of the below
    const Mat* mats = nullptr;
    struct List {
        const Tile* tiles = nullptr;
        unsigned n = 0;
    } norm, pack, gram, gram_join, poly, poly_join, apply;
    const Gap* gap = nullptr;
    int64_t gaps = 0;
};

namespace gmc {

namespace {

constexpr int64_t kMostTiles = int64_t(1) << 22;
// Tiles of 128 x 128 from which on they are taken: smaller ones read twice the bytes for each product, and
// pay where they bring more CUs to work.  X's products: 2048 x 2048 (256 tiles) 49 us, by 64 x 64 ones 62;
// 3 of 768 x 768 (108) 16 us, by 64 x 64 14.2.  G's and its square's, with their joins: 2048 x 2048 (136) 43 and
// 41 us, by 64 x 64 47 and 48; ResNet-18's matrices (about 60) 38 and 14 us, by 64 x 64 34 and 10.
constexpr int64_t kMany = 256, kManyEven = 100;
constexpr int64_t kLeastCut = 8;     // blocks of 32 columns, of a part of a contraction
constexpr int64_t kWorthCut = 48;    // by so many a tile is longer than its share for a cut to pay
constexpr int64_t kTileCost = 4;     // what a tile costs besides, in such blocks
// So many blocks for each place, cut and joined, take longer by tiles of 128 x 128 than by whole ones of 64 x 64,
// which read more: the square of ResNet-50's G's (14) 26 us and 7 for the join, by 64 x 64 26; G's own (30) 55 and 9, by 64 x 64 74.
// Of 20 plans those on either side of the border: ResNet-50's matrices (square) 822 us, so 865 without the rule; G's of 40 of
// 256 x 4096 (30) and of 2 of 1280 x 5120 (34) 854 and 1094 us, by 64 x 64 897 and 1158.  Between 14 and 30 nothing was measured.
constexpr int64_t kWorthJoin = 20;

int64_t up_to(int64_t v, int64_t step) { return (v + step - 1) / step; }

struct Part {
    int64_t offset, rows, cols, pitch;
    int64_t end() const { return offset + (rows - 1) * pitch + cols; }
};

// Over singular values s in [0, top] the largest they are taken to, and the largest |a + b s^2 + c s^4|;
// infinite where one is not finite.
struct Reach {
    double x, growth;
};

Reach reach(double a, double b, double c, double top) {
    const auto p = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
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
    Reach m = {p(top), fmax(fabs(a), slope(top))};
    for (double v : y) {
        const double s = v > 0.0 ? sqrt(v) : 0.0;
        if (s < top) {
            m.x = fmax(m.x, p(s));
            m.growth = fmax(m.growth, slope(s));
        }
    }
    if (!isfinite(m.x) || !isfinite(m.growth)) m.x = m.growth = INFINITY;
    return m;
}

// What the polynomial is held times: 2^10 (its values then stay below 61440), less where a last step takes it beyond 60.
float scale_of(double growth) {
    int half = 10;
    while (growth > 60.0 && half > -20) growth /= 2.0, --half;
    return (float)ldexp(1.0, half);
}

struct Scratch {
    _Float16 *T0, *T1, *G, *B;
    double* part;
    float *theta, *slots;
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
    s.T0 = reinterpret_cast<_Float16*>(take(p->blocks_x * 2048));
    s.T1 = reinterpret_cast<_Float16*>(take(p->blocks_x * 2048));
    s.G = reinterpret_cast<_Float16*>(take(p->blocks_g * 2048));
    s.B = reinterpret_cast<_Float16*>(take(p->blocks_g * 2048));
    s.part = reinterpret_cast<double*>(take(p->parts * 8));
    s.theta = reinterpret_cast<float*>(take(p->small ? 0 : (int64_t)p->n * (kMostSteps + 1) * 4));
    s.slots = reinterpret_cast<float*>(take(p->slots * 16384));
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
        // X and G by 2^13 have to stay below f16's 65504
        if (!(r.x <= 2.5 || (k == steps - 1 && r.x <= 1e6)))
            return op_error(GMC_EINVAL, me, "the coefficients take a singular value beyond 2.5");
        // values are kept to 2^-48 of 1, and a later step may not take that for more than it is
        if (!(r.x >= 0.25) && k < steps - 1) return op_error(GMC_EINVAL, me, "the coefficients take every singular value below 0.25");
        top = r.x;
    }
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess) return op_error(GMC_EDEVICE, me, "no current device");
    if (device != p->device) return op_error(GMC_EINVAL, me, "the plan is another device's");
    if (gmc_matrices_workspace(p)) {
        if (!workspace || workspace_bytes < gmc_matrices_workspace(p)) return op_error(GMC_EINVAL, me, "the workspace is too small");
        if (reinterpret_cast<uintptr_t>(workspace) & 255u) return op_error(GMC_EINVAL, me, "the workspace is not 256-byte aligned");
    }
    return GMC_OK;
}

// -- which workgroup does what ------------------------------------------------------

constexpr int64_t kPlaces = 512;    // workgroups of a product under way at once: two on each of 256 CUs
constexpr int kXcds = 8;

// Tiles of one matrix that share rows and columns of its operands.
struct Group {
    std::vector<Tile> tiles;
    int64_t work = 0;
};

struct Launch {
    std::vector<Tile> tiles, joins;
    int32_t slots = 0;
};

// A launch's tiles from whole ones in groups: long contractions cut where there are too few
// tiles for the places, and the groups dealt to the XCDs (workgroup b goes to XCD b % 8), each with a cache
// of its own, so that each has as much to do.
Launch deal(std::vector<Group> groups, bool may_cut) {
    Launch out;
    int64_t tiles = 0, work = 0;
    for (const Group& g : groups)
        for (const Tile& t : g.tiles) {
            ++tiles;
            work += t.last - t.first;
        }
    // a fair share of the work, and the parts each tile is cut in for it: where the wait for the longest
    // tile is shorter by more than a joining launch takes.  Equal tiles that fill the places and a few
    // more: those few are cut.
    const int64_t fair = std::max<int64_t>(kLeastCut, up_to(work, kPlaces));
    const int64_t rest = tiles > kPlaces && tiles < 4 * kPlaces ? tiles % kPlaces : 0;
    // Where most tiles are as long, a cut spares little of what the launch does at its end, and a joining
    // launch has to be worth it; where a few are long, or there is one anyway, less will do.  (Of 20 plans: with
    // kWorthCut for all, ResNet-50's matrices take 978 us for 822; with a quarter of it for all, 6 of 1024 x 1024 518 for 458,
    // 2 of 1792 x 1792 793 for 721, 5 of 1100 x 1200 594 for 518.  It is not the best for all: 2 of 1280 x 5120 take
    // 970 with the quarter for 1094, 4 of 1000 x 4096 998 for 1084.  The other 14 differ by 5 % at most.)
    int64_t long_work = 0;
    bool some = false;
    for (const Group& g : groups)
        for (const Tile& t : g.tiles) {
            if (t.last - t.first > 2 * fair) long_work += t.last - t.first;
            some = some || t.last - t.first - fair > kWorthCut;
        }
    const int64_t worth = 5 * long_work < 3 * work ? kWorthCut / 4 : some ? kWorthCut / 2 : kWorthCut;
    const auto parts_of = [&](const Tile& t, bool late) -> int32_t {
        const int64_t length = t.last - t.first;
        if (!may_cut) return 1;
        if (length - fair > worth && length >= 2 * fair) return (int32_t)(length / fair);
        if (late && length > kWorthCut) return (int32_t)std::min(kPlaces / rest, length / kLeastCut);
        return 1;
    };
    std::vector<Group> cut;
    int64_t seen = 0;
    for (Group& g : groups) {
        int32_t most = 1;
        std::vector<int32_t> count;
        for (const Tile& t : g.tiles) {
            const bool late = rest > 0 && 2 * rest <= kPlaces && seen++ >= tiles - rest;
            count.push_back(parts_of(t, late));
            most = std::max(most, count.back());
        }
        if (most < 2) {
            cut.push_back(std::move(g));
            continue;
        }
        std::vector<Group> parts(most);
        for (size_t at = 0; at < g.tiles.size(); ++at) {
            const Tile t = g.tiles[at];
            const int32_t length = t.last - t.first, n = count[at];
            Tile j = t;
            j.slot = out.slots;
            j.count = n;
            if (n > 1) {
                out.joins.push_back(j);
                out.slots += n;
            }
            for (int32_t k = 0; k < n; ++k) {
                Tile q = t;
                q.first = t.first + (int32_t)((int64_t)length * k / n);
                q.last = t.first + (int32_t)((int64_t)length * (k + 1) / n);
                q.slot = n > 1 ? j.slot + k : -1;
                parts[k].tiles.push_back(q);
            }
        }
        for (Group& q : parts)
            if (!q.tiles.empty()) cut.push_back(std::move(q));
    }
    for (Group& g : cut)
        for (const Tile& t : g.tiles) g.work += t.last - t.first + kTileCost;
    std::stable_sort(cut.begin(), cut.end(), [](const Group& a, const Group& b) { return a.work > b.work; });
    std::vector<Tile> lists[kXcds];
    int64_t load[kXcds] = {};
    for (const Group& g : cut) {
        const int x = (int)(std::min_element(load, load + kXcds) - load);
        load[x] += g.work;
        lists[x].insert(lists[x].end(), g.tiles.begin(), g.tiles.end());
    }
    size_t most = 0;
    for (auto& l : lists) {
        std::stable_sort(l.begin(), l.end(), [](const Tile& a, const Tile& b) { return a.last - a.first > b.last - b.first; });
        most = std::max(most, l.size());
    }
    for (size_t k = 0; k < most; ++k)
        for (auto& l : lists) {
            Tile none{};
            none.mat = -1;
            out.tiles.push_back(k < l.size() ? l[k] : none);
        }
    while (!out.tiles.empty() && out.tiles.back().mat < 0) out.tiles.pop_back();
    return out;
}

struct Steps {
    int32_t n;
    const double* coefficients;
    double eps;
};

// Two kernels of products: tiles of 128 x 128, and of 64 x 64 where there are few.
template <int kMode, int DT>
void run_product(int wide, dim3 grid, const ProductArgs& a, hipStream_t st) {
    if (wide == 2) matrix_product<2, 4, kMode, DT><<<grid, 256, 0, st>>>(a);
    else matrix_product<1, 3, kMode, DT><<<grid, 256, 0, st>>>(a);
}
template <int kMode>
void run_join(int wide, dim3 grid, const ProductArgs& a, hipStream_t st) {
    if (wide == 2) matrix_join<2, kMode><<<dim3(grid.x * 4), 256, 0, st>>>(a);
    else matrix_join<1, kMode><<<grid, 256, 0, st>>>(a);
}

template <int DT, bool kStep>
void run_products(const gmc_matrices* p, const Scratch& s, const Steps& how, const float* scale, ProductArgs a, hipStream_t st) {
    _Float16 *from = s.T0, *to = s.T1;
    a.slots = s.slots;
    a.G = a.Go = s.G;
    a.B = a.Bo = s.B;
    const auto take = [&](const gmc_matrices::List& l) {
        a.tiles = l.tiles;
        return dim3(l.n);
    };
    for (int32_t k = 0; k < how.n; ++k) {
        a.a = (float)how.coefficients[3 * k];
        a.b = (float)how.coefficients[3 * k + 1];
        a.c = (float)how.coefficients[3 * k + 2];
        a.scale = scale[k];
        a.XT = from;
        a.XTo = to;
        a.theta = s.theta + k;
        dim3 grid = take(p->gram);
        run_product<kGram, GMC_F32>(p->gram_wide, grid, a, st);
        if (p->gram_join.n) {
            grid = take(p->gram_join);
            run_join<kGram>(p->gram_wide, grid, a, st);
        }
        grid = take(p->poly);
        run_product<kPoly, GMC_F32>(p->poly_wide, grid, a, st);
        if (p->poly_join.n) {
            grid = take(p->poly_join);
            run_join<kPoly>(p->poly_wide, grid, a, st);
        }
        grid = take(p->apply);
        if (k + 1 < how.n) run_product<kApply, GMC_F32>(p->wide, grid, a, st);
        else if constexpr (kStep) run_product<kLastStep, GMC_F32>(p->wide, grid, a, st);
        else run_product<kLast, DT>(p->wide, grid, a, st);
        std::swap(from, to);
    }
}

template <int DT, bool kStep>
void run_steps(const gmc_matrices* p, const Scratch& s, const Steps& how, const VectorArgs& v, const ProductArgs& a, hipStream_t st) {
    VectorArgs n = v;
    n.mats = p->mats;
    n.tiles = p->norm.tiles;
    n.part = s.part;
    n.eps = how.eps;
    n.theta = s.theta;
    n.steps = how.n;
    if (p->small) n.theta = nullptr;
    double top = 1.0;
    float scale[kMostSteps];
    for (int32_t k = 0; k < how.n; ++k) {
        const Reach r = reach(how.coefficients[3 * k], how.coefficients[3 * k + 1], how.coefficients[3 * k + 2], top);
        n.growth[k] = (float)fmax(r.growth, 1.0);
        scale[k] = scale_of(r.growth);
        top = r.x;
    }
    n.XT = s.T0;
    if (p->small) {
        SmallArgs q;
        q.in = n;
        for (int32_t k = 0; k < how.n; ++k)
            for (int e = 0; e < 4; ++e) q.c[k][e] = e < 3 ? (float)how.coefficients[3 * k + e] : scale[k];
        q.out = a.out;
        q.w = a.w;
        q.alpha = a.alpha;
        q.keep = a.keep;
        q.decay = a.decay;
        const dim3 grid((unsigned)p->n);
        if (p->small == 1) matrix_small<DT, kStep, 1><<<grid, kSmallThreads, 0, st>>>(q);
        else if (p->small == 2) matrix_small<DT, kStep, 2><<<grid, kSmallThreads, 0, st>>>(q);
        else if (p->small == 3) matrix_small<DT, kStep, 3><<<grid, kSmallThreads, 0, st>>>(q);
        else matrix_small<DT, kStep, kSmallSide><<<grid, kSmallThreads, 0, st>>>(q);
        return;
    }
    matrix_norm<DT, kStep><<<dim3(p->norm.n), 256, 0, st>>>(n);
    n.tiles = p->pack.tiles;
    matrix_pack<DT, kStep><<<dim3(p->pack.n), 256, 0, st>>>(n);
    run_products<DT, kStep>(p, s, how, scale, a, st);
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
        p = new gmc_matrices;
        p->d = d;
        p->n = n;
        std::vector<Mat> mats;
        int64_t large = 0, large_even = 0;   // tiles of 128 x 128
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
            large_even += up_to(m.mb, 4) * (up_to(m.mb, 4) + 1) / 2;
            mats.push_back(m);
        }
        p->wide = large >= kMany ? 2 : 1;
        // matrices of another number of rows in blocks are padded to the most of them
        int most = 0, wide = 0;
        for (const Mat& m : mats) most = std::max(most, m.mb), wide = std::max(wide, m.nb);
        if (n > 0 && most <= kSmallSide && (int64_t)most * std::max(wide, most) + most * most <= kSmallBlocks) {
            p->small = most;
            for (Mat& m : mats) m.mb = most, m.nb = std::max(m.nb, most);
        }
        const int side = 2 * p->wide;
        std::vector<Tile> norm, pack;
        std::vector<Group> applies;
        int64_t tiles = 0;
        bool many = false;
        for (int32_t k = 0; k < n; ++k) {
            const Mat& m = mats[k];
            const int64_t mt = up_to(m.mb, side), nt = up_to(m.nb, side), mp = up_to(m.m, kSide), np = up_to(m.n, kSide);
            if (mt > kMostTiles / nt || mp > kMostTiles / np) many = true;
            else tiles += std::max(mt * nt, mp * np);
            many = many || tiles > kMostTiles;
            if (many) break;
        }
        int64_t spread = 0;   // rows that are apart
        for (const Part& q : parts) spread += q.pitch == q.cols ? 1 : q.rows;
        if (many || spread > 2 * kMostTiles) {
            delete p;
            return op_error(GMC_EINVAL, me, many ? "the matrices have more tiles than a launch takes" : "too many rows that are apart");
        }
        // the matrices' rows (dense ones' as one) in the vector's order: no two share a component, wherever they lie
        std::vector<std::pair<int64_t, int64_t>> spans;
        for (const Part& q : parts) {
            if (q.pitch == q.cols) spans.push_back({q.offset, q.rows * q.cols});
            else
                for (int64_t r = 0; r < q.rows; ++r) spans.push_back({q.offset + r * q.pitch, q.cols});
        }
        std::sort(spans.begin(), spans.end());
        for (size_t k = 1; k < spans.size(); ++k)
            if (spans[k].first < spans[k - 1].first + spans[k - 1].second) {
                delete p;
                return op_error(GMC_EINVAL, me, "two matrices share components");
            }
        for (int32_t k = 0; k < n; ++k) {
            Mat& m = mats[k];
            const int32_t mt = (m.mb + side - 1) / side, nt = (m.nb + side - 1) / side;
            const int64_t mp = up_to(m.m, kSide), np = up_to(m.n, kSide), each = up_to(mp * np, kParts);
            m.parts = (int32_t)up_to(mp * np, each);
            m.part = (int32_t)p->parts;
            p->parts += m.parts;
            for (int32_t q = 0; q < m.parts; ++q)
                norm.push_back({k, (int32_t)(q * each), q, (int32_t)std::min(each, mp * np - q * each), 0, 0, -1, 0});
            for (int32_t i = 0; i < mp; ++i)
                for (int32_t j = 0; j < np; ++j) pack.push_back({k, i, j, 1, 0, 0, -1, 0});
            // groups of up to 8 x 8 tiles, smaller ones where there are few tiles to deal out
            const int32_t most = tiles > 2048 ? 8 : 4;
            for (int32_t i0 = 0; i0 < mt; i0 += most)
                for (int32_t j0 = 0; j0 < nt; j0 += most) {
                    Group g;
                    for (int32_t j = j0; j < std::min(j0 + most, nt); ++j)
                        for (int32_t i = i0; i < std::min(i0 + most, mt); ++i) g.tiles.push_back({k, i, j, 1, 0, m.mb, -1, 0});
                    applies.push_back(std::move(g));
                }
        }
        // components between the matrices' rows
        std::vector<Gap> gap;
        int64_t at = 0, chunk = kGapChunk;
        while (d / chunk > kMostTiles / 4) chunk *= 2;
        const auto between = [&](int64_t to) {
            for (; at < to; at += chunk) gap.push_back({at, std::min(chunk, to - at)});
        };
        for (const auto& q : spans) {
            between(q.first);
            at = q.first + q.second;
        }
        between(d);
        if ((int64_t)gap.size() > 2 * kMostTiles) {
            delete p;
            return op_error(GMC_EINVAL, me, "too many pieces outside the matrices");
        }
        // the other way round than the norms: what those read last still lies in the 256 MB cache (ResNet-50's
        // step 923 us, so 916)
        std::reverse(pack.begin(), pack.end());
        // G's product or its square's: tiles with j <= i
        const auto even_groups = [&](int wide, bool square) {
            std::vector<Group> out;
            for (int32_t k = 0; k < n; ++k) {
                const int32_t even = 2 * wide, most = tiles > 2048 ? 8 : 4, et = (mats[k].mb + even - 1) / even;
                for (int32_t i0 = 0; i0 < et; i0 += most)
                    for (int32_t j0 = 0; j0 <= i0; j0 += most) {
                        Group g;
                        for (int32_t j = j0; j < std::min(j0 + most, et); ++j)
                            for (int32_t i = std::max(i0, j); i < std::min(i0 + most, et); ++i)
                                g.tiles.push_back({k, i, j, 1, 0, square ? mats[k].mb : mats[k].nb, -1, 0});
                        out.push_back(std::move(g));
                    }
            }
            return out;
        };
        const auto deal_even = [&](bool square, int& wide) {
            wide = large_even >= kManyEven ? 2 : 1;
            Launch l = deal(even_groups(wide, square), true);
            int64_t work = 0;
            for (const Tile& t : l.tiles) work += t.mat < 0 ? 0 : t.last - t.first;
            if (wide == 2 && !l.joins.empty() && work <= kWorthJoin * kPlaces) {
                Launch whole = deal(even_groups(1, square), true);
                if (whole.joins.empty()) {
                    wide = 1;
                    return whole;
                }
            }
            return l;
        };
        Launch gram, poly, apply;
        if (p->small) {   // no other launch, and nothing kept in the workspace
            norm.clear(), pack.clear();
            p->blocks_x = p->blocks_g = p->parts = 0;
        } else {
            gram = deal_even(false, p->gram_wide);
            poly = deal_even(true, p->poly_wide);
            apply = deal(std::move(applies), false);
        }
        p->slots = std::max((int64_t)gram.slots * p->gram_wide * p->gram_wide, (int64_t)poly.slots * p->poly_wide * p->poly_wide);
        std::vector<char> host;
        const auto add = [&](const void* from, size_t bytes) {
            const size_t here = host.size();
            host.resize(here + (bytes + 255) / 256 * 256);
            if (bytes) memcpy(host.data() + here, from, bytes);
            return here;
        };
        const std::vector<Tile>* lists[] = {&norm, &pack, &gram.tiles, &gram.joins, &poly.tiles, &poly.joins, &apply.tiles};
        gmc_matrices::List* said[] = {&p->norm, &p->pack, &p->gram, &p->gram_join, &p->poly, &p->poly_join, &p->apply};
        size_t at_list[7];
        const size_t at_mats = add(mats.data(), mats.size() * sizeof(Mat));
        for (int k = 0; k < 7; ++k) at_list[k] = add(lists[k]->data(), lists[k]->size() * sizeof(Tile));
        const size_t at_gap = add(gap.data(), gap.size() * sizeof(Gap));
        p->gaps = gap.size();
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
        for (int k = 0; k < 7; ++k) {
            said[k]->tiles = reinterpret_cast<const Tile*>(t + at_list[k]);
            said[k]->n = (unsigned)lists[k]->size();
        }
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
    if (plan->table) {
        int current = plan->device;
        (void)hipGetDevice(&current);
        const bool waited = hipSetDevice(plan->device) == hipSuccess && hipDeviceSynchronize() == hipSuccess;
        // (no table is freed that a call may still read)
        if (!waited || hipFree(plan->table) != hipSuccess) (void)hipGetLastError();
        if (current != plan->device) (void)hipSetDevice(current);
    }
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
    const Span x(x_dev, bytes), out(out_dev, bytes), scratch(workspace_dev, gmc_matrices_workspace(plan));
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
        out(w_out_dev, plan->d * 4), scratch(workspace_dev, gmc_matrices_workspace(plan));
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
            // decays beyond a half leave less than they take: 1 - decay is the small one
            const bool small = fabs(decay) <= 0.5;
            a.keep = small ? 1.0f : (float)(1.0 - decay);
            a.decay = small ? (float)decay : 0.0f;
            run_steps<DT, true>(plan, layout(plan, workspace_dev), {steps, coefficients, eps}, v, a, st);
        }
    });
    return op_launched(me);
}

}  // extern "C"
