// Dropout with a mask that is never stored, with or without the residual add,
// forward and backward (gmc_dropout in include/gmc.h).
//
// Mask: element i of the activations, counted over rows and columns, takes bits
// 16 (i mod 4) .. 16 (i mod 4) + 15 of draw i / 4 of a SplitMix64 stream whose
// state comes from (seed, t, worker, site); it is kept when they reach level =
// round(65536 p).  The mask is a function of the element's number alone, so the
// backward pass draws it again, whatever the layouts.  16 bits an element, not
// 32: the two 64-bit products of a draw are then shared by four elements, about 12
// operations each, which the stream hides.  Bound by memory: 16384 x 768 bf16 with the
// residual 12 us (6.0 TB/s), 65536 x 4096 286 us (5.6); its smallest calls by the host
// (one launch, 7 us with the binding's part).  Nontemporal accesses or runs of blocks
// per XCD gain nothing below half a gigabyte (52 us become 57 to 61 at 65536 x 768).
#include <math.h>

#include "gmc_ops.h"

namespace gmc {

namespace {

constexpr uint64_t kGamma = 0x9e3779b97f4a7c15ull;
constexpr int kDropThreads = 256;

// The output mix of SplitMix64 (Steele, Lea and Flood, OOPSLA 2014).
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
    z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
    return z ^ (z >> 31);
}

struct DropArgs {
    const void* x;
    const void* r;
    void* y;
    int64_t x_pitch, r_pitch, y_pitch;
    int64_t cols, vecs, total;  // vecs: vectors per row; total: rows * vecs
    uint64_t state;
    uint32_t level;
    float scale;  // 65536 / (65536 - level), 0 when nothing is kept
};

// y = (kept ? x scale : 0) [+ r] for N elements starting at element i.  The
// product and the sum are 32-bit; the caller rounds once.
template <int N, bool kAdd>
__device__ __forceinline__ void drop(const DropArgs& a, uint64_t i, const float (&x)[N], const float (&r)[N],
                                     float (&y)[N]) {
    const uint32_t o = 16u * ((uint32_t)i & 3u);
    uint64_t s = a.state + ((i >> 2) + 1) * kGamma;
    uint64_t w = mix64(s);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
        uint64_t bits = w;
        if (o) {  // the elements straddle draws
            s += kGamma;
            w = mix64(s);
            bits = (bits >> o) | (w << (64u - o));
        } else if (q + 1 < N / 4) {
            s += kGamma;
            w = mix64(s);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t b = (uint32_t)(bits >> (16 * e)) & 0xffffu;
            const float v = b >= a.level ? x[4 * q + e] * a.scale : 0.0f;
            y[4 * q + e] = kAdd ? r[4 * q + e] + v : v;
        }
    }
}

// Vectors of 16 bytes, kUnroll a thread, their loads issued together; a row's
// last elements one by one.
template <int DT, bool kAdd, int kUnroll>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int N = 16 / Elem<DT>::kSize;
    typedef Vec<DT, N> V;
    const T* px = static_cast<const T*>(a.x);
    const T* pr = static_cast<const T*>(a.r);
    T* py = static_cast<T*>(a.y);
    const int64_t first = (int64_t)blockIdx.x * (kDropThreads * kUnroll) + threadIdx.x;
    V xv[kUnroll], rv[kUnroll];
    int64_t row[kUnroll], col[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t q = first + u * kDropThreads;
        if (a.vecs == a.total) {
            row[u] = 0;
            col[u] = q * N;
        } else if (a.total <= 0x7fffffff) {
            row[u] = (uint32_t)q / (uint32_t)a.vecs;
            col[u] = ((uint32_t)q - (uint32_t)row[u] * (uint32_t)a.vecs) * (int64_t)N;
        } else {
            row[u] = q / a.vecs;
            col[u] = (q - row[u] * a.vecs) * N;
        }
        if (q < a.total && col[u] + N <= a.cols) {
            xv[u] = V::load(px + row[u] * a.x_pitch + col[u]);
            if (kAdd) rv[u] = V::load(pr + row[u] * a.r_pitch + col[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        if (first + u * kDropThreads >= a.total) return;
        const uint64_t i = (uint64_t)row[u] * (uint64_t)a.cols + (uint64_t)col[u];
        T* out = py + row[u] * a.y_pitch + col[u];
        float x[N], r[N], y[N];
        if (col[u] + N <= a.cols) {
            xv[u].unpack(x);
            if (kAdd) rv[u].unpack(r);
            drop<N, kAdd>(a, i, x, r, y);
            xv[u].pack(y);
            xv[u].store(out);
        } else {
            const int n = (int)(a.cols - col[u]);
            const T* xs = px + row[u] * a.x_pitch + col[u];
            const T* rs = pr + row[u] * a.r_pitch + col[u];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = e < n ? Elem<DT>::up(xs[e]) : 0.0f;
                r[e] = kAdd && e < n ? Elem<DT>::up(rs[e]) : 0.0f;
            }
            drop<N, kAdd>(a, i, x, r, y);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e < n) out[e] = Elem<DT>::down(y[e]);
        }
    }
}

}  // namespace

}  // namespace gmc

using namespace gmc;

extern "C" gmc_status gmc_dropout(void* hip_stream, int32_t dtype, int64_t rows, int64_t cols, const void* x_dev,
                                  int64_t x_pitch, const void* residual_dev, int64_t residual_pitch, void* y_dev,
                                  int64_t y_pitch, double p, uint64_t seed, int64_t t, int32_t worker, int32_t site) {
    const char* me = "gmc_dropout";
    if (!known_type(dtype)) return op_error(GMC_EINVAL, me, "unknown element type");
    if (rows < 0 || cols < 0) return op_error(GMC_EINVAL, me, "rows and cols must be >= 0");
    if (!(p >= 0.0 && p <= 1.0)) return op_error(GMC_EINVAL, me, "p must be in [0, 1]");
    if (t < 0 || worker < 0 || worker >= GMC_MAX_WORKERS || site < 0)
        return op_error(GMC_EINVAL, me, "need t >= 0, 0 <= worker < 64, site >= 0");
    if (rows == 0 || cols == 0) return GMC_OK;
    if (!x_dev || !y_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    if (rows > 1 && (x_pitch < cols || y_pitch < cols || (residual_dev && residual_pitch < cols)))
        return op_error(GMC_EINVAL, me, "a row pitch is shorter than a row");
    constexpr int64_t kMost = int64_t(1) << 40;
    if (rows > kMost || cols > kMost || rows > kMost / cols || x_pitch > kMost / rows || y_pitch > kMost / rows ||
        (residual_dev && residual_pitch > kMost / rows))
        return op_error(GMC_EINVAL, me, "more than 2^40 elements");
    const int64_t b = type_size(dtype);
    const auto span = [&](int64_t pitch) { return ((rows - 1) * pitch + cols) * b; };
    // in place is one thread reading and then writing the same element
    const bool same_x = x_dev == y_dev && x_pitch == y_pitch;
    const bool same_r = residual_dev == y_dev && residual_pitch == y_pitch;
    if ((!same_x && overlap(x_dev, span(x_pitch), y_dev, span(y_pitch))) ||
        (residual_dev && !same_r && overlap(residual_dev, span(residual_pitch), y_dev, span(y_pitch))))
        return op_error(GMC_EINVAL, me, "y overlaps an input without being it");
    DropArgs a{};
    a.x = x_dev;
    a.r = residual_dev;
    a.y = y_dev;
    a.x_pitch = x_pitch;
    a.r_pitch = residual_pitch;
    a.y_pitch = y_pitch;
    if (rows > 1 && x_pitch == cols && y_pitch == cols && (!residual_dev || residual_pitch == cols)) {
        cols *= rows;  // one row
        rows = 1;
    }
    const int64_t n = 16 / b;
    a.cols = cols;
    a.vecs = (cols + n - 1) / n;
    a.total = rows * a.vecs;
    a.state = seed ^ mix64((uint64_t)t + 1) ^ mix64((uint64_t)(worker + 1) << 32 | (uint64_t)((uint32_t)site + 1u));
    a.level = (uint32_t)floor(p * 65536.0 + 0.5);
    a.scale = a.level == 65536u ? 0.0f : (float)(65536.0 / (65536.0 - (double)a.level));
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    // one vector a thread until that gives every CU several workgroups
    const int64_t unroll = a.total >= int64_t(kDropThreads) * 4 * 2048 ? 4 : 1;
    const int64_t blocks = (a.total + kDropThreads * unroll - 1) / (kDropThreads * unroll);
    if (blocks > 0xffffffffll / kDropThreads) return op_error(GMC_EINVAL, me, "too many vectors for one launch");
    const dim3 grid((unsigned)blocks);
    GMC_BY_TYPE(dtype, {
        if (a.r) {
            if (unroll == 4) dropout_kernel<DT, true, 4><<<grid, kDropThreads, 0, st>>>(a);
            else dropout_kernel<DT, true, 1><<<grid, kDropThreads, 0, st>>>(a);
        } else {
            if (unroll == 4) dropout_kernel<DT, false, 4><<<grid, kDropThreads, 0, st>>>(a);
            else dropout_kernel<DT, false, 1><<<grid, kDropThreads, 0, st>>>(a);
        }
    });
    return op_launched(me);
}
