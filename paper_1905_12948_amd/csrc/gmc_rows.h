// What the operators on rows of logits (gmc_loss.hip, gmc_scores.hip) share: which
// row a workgroup takes, a row as vectors and edges, and the checks of the logits' and
// labels' arguments.  Not part of the ABI.
#pragma once

#include <math.h>

#include "gmc_ops.h"

namespace gmc {

namespace {

// The row of a workgroup, or of a wavefront where four share one; the same value
// in every lane, so that what follows from it stays in scalar registers.  The
// workgroups go to the 8 XCDs in turn; each XCD takes a run of neighbouring rows
// (a plain copy of 100 KB rows: 5.9 TB/s, in the launch's order 5.6).
template <int kThreads>
__device__ __forceinline__ int64_t row_of() {
    const int64_t id = xcd_run(blockIdx.x, gridDim.x);
    if constexpr (kThreads == 64) return id * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    else return id;
}

// A row of V elements as a head and a tail of single elements and a body of
// vectors.  The body begins where the row that is written (where only the logits
// are read, that one), `at` elements from the start of its tensor, crosses a line, or
// 16 bytes where a wavefront has a row of its own: a wavefront's accesses then cover
// whole lines; with lines split between two of them the copy above takes 5% longer.
// It follows the pitches, not the pointers, so that a row's sums have one order
// wherever the tensors lie.
template <int DT, int kThreads>
struct Row {
    typedef typename Elem<DT>::T T;
    static constexpr int kSize = Elem<DT>::kSize;
    static constexpr int N = 16 / kSize;
    static constexpr int kAlign = kThreads == 64 ? 16 : 128;
    const T* p;
    int V, head, nb, tail;

    __device__ __forceinline__ Row(const T* q, int v, int64_t at) : p(q), V(v) {
        constexpr int kStep = kAlign / kSize;
        const int off = (int)(at & (kStep - 1));
        head = off ? kStep - off : 0;
        if (head > V) head = V;
        nb = (V - head) / N;
        tail = V - head - nb * N;
    }
    // The index of thread `tid`'s single element, -1 for most threads.
    __device__ __forceinline__ int edge(int tid) const {
        constexpr int kTail = kThreads == 64 ? 32 : 64;
        if (tid < head) return tid;
        if (tid >= kTail && tid < kTail + tail) return V - tail + (tid - kTail);
        return -1;
    }
};

// A vector of -inf.
template <int DT, int N>
__device__ __forceinline__ Vec<DT, N> nothing() {
    Vec<DT, N> v;
    const uint32_t w = DT == GMC_F32 ? 0xff800000u : DT == GMC_BF16 ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
    for (int i = 0; i < Vec<DT, N>::kBytes / 4; ++i) v.set_word(i, w);
    return v;
}

// Zeros over a row whose first element is `at` elements from the start of its tensor.
template <int DT, int kThreads>
__device__ __forceinline__ void zero_row(typename Elem<DT>::T* out, int V, int64_t at, int tid) {
    const Row<DT, kThreads> row(out, V, at);
    constexpr int N = row.N;
    Vec<DT, N> z;
    const float f[N] = {};
    z.pack(f);
    for (int v = tid; v < row.nb; v += kThreads) z.store_once(out + row.head + (int64_t)v * N);
    const int e = row.edge(tid);
    if (e >= 0) out[e] = Elem<DT>::down(0.0f);
}

constexpr int64_t kMostRows = 0xffffffffll / 1024;

inline bool finite_f32(double v) { return isfinite((float)v); }

// The bytes of R sequences of T rows of V elements of b bytes.
inline int64_t rows_span(int64_t R, int64_t T, int64_t V, int64_t seq, int64_t tok, int64_t b) {
    return ((R - 1) * (R > 1 ? seq : 0) + (T - 1) * (T > 1 ? tok : 0) + V) * b;
}

// What a call on logits refuses; labels may be missing where `unlabelled` says so.
inline gmc_status logits_check(const char* me, int32_t dtype, int64_t R, int64_t T, int64_t V, const void* logits,
                               int64_t seq, int64_t tok, const void* grad, int64_t grad_seq, int64_t grad_tok,
                               const void* labels, int64_t label_pitch, bool unlabelled = false) {
    if (!known_type(dtype)) return op_error(GMC_EINVAL, me, "unknown element type");
    if (R < 0 || T < 0 || V < 1 || V > 0x3fffffff)
        return op_error(GMC_EINVAL, me, "need R >= 0, T >= 0 and 1 <= V < 2^30");
    if (R == 0 || T == 0) return GMC_OK;
    if (R > kMostRows / T) return op_error(GMC_EINVAL, me, "more than 2^22 - 1 tokens");
    if (!logits || (!labels && !unlabelled)) return op_error(GMC_EINVAL, me, "NULL argument");
    const auto fits = [&](int64_t s, int64_t k) {
        constexpr int64_t kMost = int64_t(1) << 50;
        if (T > 1 && (k < V || k > kMost / T)) return false;
        return R == 1 || (s >= (T - 1) * (T > 1 ? k : 0) + V && s <= kMost / R);
    };
    if (!fits(seq, tok) || (grad && !fits(grad_seq, grad_tok)))
        return op_error(GMC_EINVAL, me, "a pitch is shorter than what it steps over");
    if (labels && R > 1 && (label_pitch < T || label_pitch > (int64_t(1) << 50) / R))
        return op_error(GMC_EINVAL, me, "the label pitch is shorter than a row");
    if (grad) {
        const int64_t b = type_size(dtype);
        const bool same = logits == grad && (R == 1 || seq == grad_seq) && (T == 1 || tok == grad_tok);
        if (!same && overlap(logits, rows_span(R, T, V, seq, tok, b), grad, rows_span(R, T, V, grad_seq, grad_tok, b)))
            return op_error(GMC_EINVAL, me, "the gradient overlaps the logits without being them");
    }
    return GMC_OK;
}

}  // namespace

}  // namespace gmc
