// The clipped policy loss with its KL term and the preference loss, from logits,
// with the logits' gradient (gmc_policy_loss and gmc_preference_loss in
// include/gmc.h).
//
// Both gradients have the form  dlogits_j = c (delta_jy - p_j)  with p the
// token's softmax and c a scalar of the token.  A row of logits is a token's
// vocabulary; with e_j = 2^((x_j - b) L), L = log2(e) / tau, and s = sum e_j for
// any shift b:  log p_y = ((x_y - b) L - log2 s) ln 2  and  c p_j = (c / s) e_j.
//
// The shift: b = 0 while s stays within [2^-40, 2^60], where every e_j that
// counts is a normal number and no value has been lost; this spares a pass for
// the maximum.  A row outside that range (logits beyond about 40 or all below
// about -27, infinities, NaN) is taken again with b its maximum, for which any
// finite logits are in range (rows at the type's lowest value among them); -inf
// entries give zeros either way.
//
// Policy: c depends on the token alone, so a workgroup keeps the row in its
// registers: the logits are read once and the gradient is written once, the
// floor of the bytes.  16 x 1024 x 50257 bf16, three quarters of the tokens counting:
// 504 us, 5.7 TB/s, where a plain copy of such rows reaches 5.9; 555 us from a view
// whose rows lie off the gradient's by other than 16 bytes.  Beyond 6,656 vectors
// (53,248 entries of 16 bits) a thread's share of the row leaves too few registers for
// the rest: 43 of 128 go through scratch memory at 26 vectors of 512 threads, 8 at 20 of
// 1024, with 5.0 to 5.3 TB/s from 53,256 to 151,936 bf16 entries.  Longer rows than 20,480
// vectors are read twice (200,000: 4.8 TB/s of one read and the write).  Preference: c needs the
// pair's sums over all its tokens; the rows are read for the statistics and again for
// the gradient, 16 x 512 tokens of which two thirds count in 301 us.  Both are bound by
// memory: an exponential and its conversions take about 15 operations an element, 40%
// of what the vector units give in that time.
// Ignored tokens' logits are never read, and their gradient is zero.
#include <math.h>

#include <type_traits>

#include "gmc_ops.h"

namespace gmc {

namespace {

constexpr int kFinishBlocks = 32;     // workgroups that add the tokens' shares of the loss
constexpr int64_t kFewTokens = 65536, kFewSequences = 256;  // counted by one workgroup
constexpr int64_t kRowPairs = 8, kRowPairTokens = 512;  // pairs worked out with every row
constexpr int64_t kRowTokens = 2048;  // counted by every row's workgroup
constexpr int kLongest = 20;         // vectors each of 1024 threads holds of the longest held row
constexpr int kRowThreads = 1024;    // rows that no workgroup's registers hold
constexpr int kStatThreads = 256;    // preference rows
constexpr float kLeast = 0x1p-40f, kGreatest = 0x1p60f;  // a sum of unshifted e_j in range

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

// Workgroup-wide (max, sum of 2^((x - max) L)) from every thread's own; one
// barrier, every thread gets the result.  kWaves = 1: a wavefront's own row.
template <int kWaves>
__device__ __forceinline__ void join_stats(float L, float& m, float& s, float2* lds) {
    const float wm = wave_max(m);
    const float base = wm == -INFINITY ? 0.0f : wm;
    s = wave_sum(s * exp2_fast((m - base) * L));
    m = wm;
    if (kWaves == 1) return;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(m, s);
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds[w].x);
    const float b = top == -INFINITY ? 0.0f : top;
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += lds[w].y * exp2_fast((lds[w].x - b) * L);
    m = top;
    s = t;
}

// The sum over the row's threads, in every thread, and that of a number each
// wavefront brings; one barrier.
template <int kWaves>
__device__ __forceinline__ float row_sum(float s, int& n, float2* lds) {
    s = wave_sum(s);
    if (kWaves == 1) return s;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(s, __int_as_float(n));
    __syncthreads();
    s = 0.0f;
    n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        s += lds[w].x;
        n += __float_as_int(lds[w].y);
    }
    return s;
}

__device__ __forceinline__ bool in_range(float s) { return s >= kLeast && s <= kGreatest; }

// Unshifted e_j of a vector.
template <int N>
__device__ __forceinline__ void exps(float (&f)[N], float L) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = exp2_fast(f[i] * L);
}

// e_j of a vector, the maximum subtracted.
template <int N>
__device__ __forceinline__ void exps(float (&f)[N], float base, float L) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = exp2_fast((f[i] - base) * L);
}

// (max, sum) over the thread's share of a row, read in passes of four vectors.
template <int DT, int kThreads>
__device__ __forceinline__ void stream_stats(const Row<DT, kThreads>& row, int tid, float L, float& m, float& s) {
    constexpr int N = 16 / Elem<DT>::kSize;
    typedef Vec<DT, N> V;
    m = -INFINITY;
    s = 0.0f;
    const int e = row.edge(tid);
    if (e >= 0) {
        m = Elem<DT>::up(row.p[e]);
        s = m == -INFINITY ? 0.0f : m == m && m < INFINITY ? 1.0f : NAN;
    }
    for (int v0 = tid; v0 < row.nb; v0 += 4 * kThreads) {
        V x[4];
        float f[N];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (v0 + k * kThreads < row.nb) x[k] = V::load_once(row.p + row.head + (int64_t)(v0 + k * kThreads) * N);
        float cm = m;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (v0 + k * kThreads < row.nb) {
                x[k].unpack(f);
#pragma unroll
                for (int i = 0; i < N; ++i) cm = fmaxf(cm, f[i]);
            }
        const float base = cm == -INFINITY ? 0.0f : cm;
        s *= exp2_fast((m - base) * L);
        m = cm;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (v0 + k * kThreads < row.nb) {
                x[k].unpack(f);
                exps<N>(f, base, L);
#pragma unroll
                for (int i = 0; i < N; ++i) s += f[i];
            }
    }
}

// A vector of the gradient: c (delta - p), k = -c / s, at = the label's place
// in it or outside [0, N).
template <int N, bool kShift>
__device__ __forceinline__ void gradient(float (&f)[N], float base, float L, float k, float c, int at) {
    if constexpr (kShift) exps<N>(f, base, L);
    else exps<N>(f, L);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = f[i] * k;
    if ((unsigned)at < (unsigned)N)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i == at) f[i] += c;
}

// A vector of -inf.
template <int DT, int N>
__device__ __forceinline__ Vec<DT, N> nothing() {
    Vec<DT, N> v;
    const uint32_t w = DT == GMC_F32 ? 0xff800000u : DT == GMC_BF16 ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
    for (int i = 0; i < Vec<DT, N>::kBytes / 4; ++i) v.set_word(i, w);
    return v;
}

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

// The gradient of a row read from memory, element by element in its own thread
// (so it may be written over the logits).
template <int DT, int kThreads, bool kShift>
__device__ __forceinline__ void stream_gradient(const Row<DT, kThreads>& row, typename Elem<DT>::T* out, int tid,
                                                float base, float L, float k, float c, int y) {
    constexpr int N = 16 / Elem<DT>::kSize;
    constexpr int threads = kThreads;
    typedef Vec<DT, N> V;
    for (int v0 = tid; v0 < row.nb; v0 += 4 * threads) {
        V x[4];
        float f[N];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (v0 + u * threads < row.nb) x[u] = V::load_once(row.p + row.head + (int64_t)(v0 + u * threads) * N);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (v0 + u * threads < row.nb) {
                const int j = row.head + (v0 + u * threads) * N;
                x[u].unpack(f);
                gradient<N, kShift>(f, base, L, k, c, y - j);
                x[u].pack(f);
                x[u].store_once(out + j);
            }
    }
    const int e = row.edge(tid);
    if (e >= 0) {
        float f[1] = {Elem<DT>::up(row.p[e])};
        gradient<1, kShift>(f, base, L, k, c, y - e);
        out[e] = Elem<DT>::down(f[0]);
    }
}

// The gradient of the row `in` with shift and sum st, in place or not.
template <int DT, int kThreads>
__device__ __forceinline__ void write_gradient(const typename Elem<DT>::T* in, typename Elem<DT>::T* out, int V,
                                               int64_t at, int tid, float2 st, float L, float c, int y) {
    const Row<DT, kThreads> row(in, V, at);
    if (st.x == 0.0f) stream_gradient<DT, kThreads, false>(row, out, tid, 0.0f, L, -c / st.y, c, y);
    else stream_gradient<DT, kThreads, true>(row, out, tid, st.x == -INFINITY ? 0.0f : st.x, L, -c / st.y, c, y);
}

// A row's shift and sum, read from memory: (0, s) in range, else with the maximum.
// kOnce: nothing reads the row again.
template <int DT, int kThreads, bool kOnce>
__device__ __forceinline__ float2 stream_row(const Row<DT, kThreads>& row, int tid, float L, float2* lds) {
    constexpr int N = 16 / Elem<DT>::kSize;
    constexpr int kWaves = kThreads / 64;
    constexpr int kBatch = 8;
    typedef Vec<DT, N> V;
    const int e = row.edge(tid);
    float s = e >= 0 ? exp2_fast(Elem<DT>::up(row.p[e]) * L) : 0.0f;
    for (int v0 = tid; v0 < row.nb; v0 += kBatch * kThreads) {
        V x[kBatch];
        float f[N];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (v0 + k * kThreads < row.nb) {
                const typename Elem<DT>::T* q = row.p + row.head + (int64_t)(v0 + k * kThreads) * N;
                x[k] = kOnce ? V::load_once(q) : V::load(q);
            }
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (v0 + k * kThreads < row.nb) {
                x[k].unpack(f);
                exps<N>(f, L);
#pragma unroll
                for (int i = 0; i < N; ++i) s += f[i];
            }
    }
    int none = 0;
    s = row_sum<kWaves>(s, none, lds);
    if (in_range(s)) return make_float2(0.0f, s);
    float m;
    stream_stats<DT, kThreads>(row, tid, L, m, s);
    if (kWaves > 1) __syncthreads();  // the sums are read
    join_stats<kWaves>(L, m, s, lds);
    return make_float2(m, s);
}

// log p_y of a row with shift M (-inf: all entries are) and sum s.  Of log2 s =
// k + log2 f only the second part, of size below 1, is rounded to 32 bits; the rest
// is in 64, so that what is taken from it, such as a ratio to an old log-probability
// near it, does not lose the bits that cancel.
__device__ __forceinline__ double logp_of(float xy, float M, float L, float s) {
    const float base = M == -INFINITY ? 0.0f : M;
    int k;
    const float f = frexpf(s, &k);
    return (((double)xy - (double)base) * (double)L - (double)k - (double)__log2f(f)) * 0.69314718055994531;
}

// -- policy -------------------------------------------------------------------

struct PolicyArgs {
    const void* logits;
    void* grad;  // NULL: the loss alone
    int64_t seq, tok, grad_seq, grad_tok;
    const int64_t* labels;
    int64_t label_pitch, ignore;
    const float* old_logp;  // NULL: the present ones
    const float* ref_logp;  // NULL: no KL term
    const float* adv;
    int64_t adv_seq, adv_tok;
    int64_t R, T, rows;
    int32_t V;
    float lo, hi, kl, L, inv_tau, scale;
    int32_t by_sequence;
    float* logp;
    const float* weight;  // policy_weight's; NULL: the mean over few tokens, counted with each row
    float4* tokens;       // per token: weighted loss, KL, clipped
    double* sums;         // [3][kFinishBlocks]
    int* done;            // workgroups of the last launch that have added theirs
    float* stats;
};

// Weights of the mean over tokens, or of the mean over sequences of their means:
// weight[0] the reciprocal of all tokens that count, or of the sequences with any;
// weight[1 + r] the tokens of sequence r.  One workgroup, a wavefront a sequence at
// a time, four loads in flight; with many tokens the sequences are counted first by
// a launch of their own.
__device__ __forceinline__ int count_labels(const int64_t* labels, int64_t T, int64_t ignore) {
    int n = 0;
#pragma unroll 4
    for (int64_t t = threadIdx.x & 63; t < T; t += 64) n += labels[t] != ignore;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    return n;
}

__global__ __launch_bounds__(256) void policy_counts(PolicyArgs a, float* weight) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= a.R) return;
    const int n = count_labels(a.labels + r * a.label_pitch, a.T, a.ignore);
    if ((threadIdx.x & 63) == 0) weight[1 + r] = (float)n;
}

template <bool kCounted>
__global__ __launch_bounds__(1024) void policy_weight(PolicyArgs a, float* weight) {
    __shared__ double lds[16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    double n = 0.0;
    if constexpr (kCounted) {
        for (int64_t r = threadIdx.x; r < a.R; r += 1024) {
            const float c = weight[1 + r];
            n += a.by_sequence ? (c > 0.0f ? 1.0 : 0.0) : (double)c;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    } else {
        for (int64_t r = wave; r < a.R; r += 16) {
            const int c = count_labels(a.labels + r * a.label_pitch, a.T, a.ignore);
            if (lane == 0) weight[1 + r] = (float)c;
            n += a.by_sequence ? (c > 0 ? 1.0 : 0.0) : (double)c;
        }
    }
    if (lane == 0) lds[wave] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < 16; ++w) t += lds[w];
        weight[0] = t > 0.0 ? (float)(1.0 / t) : 0.0f;
        *a.done = 0;
    }
}

// A token's inputs, loaded ahead of the row's sum.
struct Token {
    float w, A, old, ref;
};

__device__ __forceinline__ Token policy_token(const PolicyArgs& a, int64_t r, int64_t t) {
    Token k;
    k.w = !a.weight ? 0.0f : a.by_sequence ? a.weight[0] / a.weight[1 + r] : a.weight[0];
    k.A = a.adv[r * a.adv_seq + t * a.adv_tok];
    k.old = a.old_logp ? a.old_logp[r * a.T + t] : 0.0f;
    k.ref = a.ref_logp ? a.ref_logp[r * a.T + t] : 0.0f;
    return k;
}

// The tokens that count, of those this wavefront looks at.
__device__ __forceinline__ int count_tokens(const PolicyArgs& a, int tid, int threads) {
    int n = 0;
    for (int i0 = 0; i0 < (int)a.rows; i0 += threads) {
        const int i = i0 + tid;
        bool some = false;
        if (i < (int)a.rows) {
            const int r = i / (int)a.T;
            some = a.labels[r * a.label_pitch + (i - r * (int)a.T)] != a.ignore;
        }
        n += __popcll(__ballot(some));
    }
    return n;
}

// What the clipped term is: the ratio's product, the smaller of the two, and
// whether that is the unclipped one, which the gradient follows.
struct Clip {
    float unclipped, smaller;
    bool free;
};

__device__ __forceinline__ Clip policy_clip(const PolicyArgs& a, const Token& k, double logp) {
    float ratio = a.old_logp ? exp2_fast((float)(logp - k.old) * kLog2e) : logp == logp ? 1.0f : NAN;
    // beyond 32 bits, from an old log-probability far below: a token without advantage adds 0 all the same
    if (k.A == 0.0f && ratio == INFINITY) ratio = 1.0f;
    Clip c;
    c.unclipped = ratio * k.A;
    const float clipped = fminf(fmaxf(ratio, 1.0f - a.lo), 1.0f + a.hi) * k.A;
    c.free = !(c.unclipped > clipped);
    c.smaller = c.free ? c.unclipped : clipped;
    return c;
}

// c: the loss's slope in the logits' log-probability, for the gradient.
__device__ __forceinline__ float policy_slope(const PolicyArgs& a, const Token& k, double logp) {
    const Clip c = policy_clip(a, k, logp);
    float slope = c.free ? -c.unclipped : 0.0f;
    if (a.ref_logp && a.kl != 0.0f) slope = __builtin_fmaf(-a.kl, expm1f((float)(k.ref - logp)), slope);
    return a.scale * a.inv_tau * k.w * slope;
}

// What the token adds to the loss, by one thread.
__device__ __forceinline__ void policy_write(const PolicyArgs& a, int64_t i, const Token& k, double logp) {
    const Clip c = policy_clip(a, k, logp);
    float kl = 0.0f;
    if (a.ref_logp) {
        const float d = (float)(k.ref - logp);
        kl = expm1f(d) - d;
    }
    a.logp[i] = (float)logp;
    // without a coefficient the term is not in the loss, be it beyond 32 bits
    a.tokens[i] = make_float4(k.w * (-c.smaller + (a.kl != 0.0f ? a.kl * kl : 0.0f)), k.w * kl, c.free ? 0.0f : k.w, 0.0f);
}

// A row's label, its logit (NaN where the label is out of range) and place (-1).
template <int DT>
struct Label {
    int y;
    float x;
    __device__ __forceinline__ Label(const typename Elem<DT>::T* row, int V, int64_t label) {
        const bool known = (uint64_t)label < (uint64_t)V;
        y = known ? (int)label : -1;
        x = known ? Elem<DT>::up(row[y]) : NAN;
    }
};

template <int DT, int kThreads>
__device__ __forceinline__ void policy_ignored(const PolicyArgs& a, int64_t i, int64_t at, int tid) {
    if (tid == 0) {
        a.logp[i] = 0.0f;
        a.tokens[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    if (a.grad) zero_row<DT, kThreads>(static_cast<typename Elem<DT>::T*>(a.grad) + at, a.V, at, tid);
}

// One row of logits per kThreads threads, held in kHeld vectors a thread.
template <int DT, int kThreads, int kHeld>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) __attribute__((amdgpu_waves_per_eu(kHeld <= 8 ? 6 : 4)))
void policy_held(PolicyArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int N = 16 / Elem<DT>::kSize;
    constexpr int kWaves = kThreads / 64;
    typedef Vec<DT, N> V;
    __shared__ float2 lds[kWaves];
    const int tid = threadIdx.x % kThreads;
    const int64_t i = row_of<kThreads>();
    if (i >= a.rows) return;
    const int64_t r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels[r * a.label_pitch + t];
    const int64_t at = r * a.grad_seq + t * a.grad_tok;
    T* out = static_cast<T*>(a.grad) + at;
    if (label == a.ignore) {
        policy_ignored<DT, kThreads>(a, i, at, tid);
        return;
    }
    const T* in = static_cast<const T*>(a.logits) + r * a.seq + t * a.tok;
    const Row<DT, kThreads> row(in, a.V, at);
    // past the row's end a vector holds -inf, so that only loads and stores ask for the end
    V x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (k * kThreads < row.nb) {
            x[k] = nothing<DT, N>();
            if (tid + k * kThreads < row.nb) x[k] = V::load_once(row.p + row.head + (int64_t)(tid + k * kThreads) * N);
        }
    const int e = row.edge(tid);
    const float ex = e >= 0 ? Elem<DT>::up(row.p[e]) : -INFINITY;
    const Label<DT> lab(in, a.V, label);
    Token tk = policy_token(a, r, t);
    int kept = a.weight ? 0 : count_tokens(a, tid, kThreads);
    float f[N], s = exp2_fast(ex * a.L), base = 0.0f;
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (k * kThreads < row.nb) {
            x[k].unpack(f);
            exps<N>(f, a.L);
#pragma unroll
            for (int q = 0; q < N; ++q) s += f[q];
        }
    s = row_sum<kWaves>(s, kept, lds);
    if (!a.weight) tk.w = 1.0f / (float)kept;
    const bool shifted = !in_range(s);
    if (shifted) {
        float m = ex;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (k * kThreads < row.nb) {
                x[k].unpack(f);
#pragma unroll
                for (int q = 0; q < N; ++q) m = fmaxf(m, f[q]);
            }
        m = wave_max(m);
        const float own = m == -INFINITY ? 0.0f : m;
        s = exp2_fast((ex - own) * a.L);
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (k * kThreads < row.nb) {
                x[k].unpack(f);
                exps<N>(f, own, a.L);
#pragma unroll
                for (int q = 0; q < N; ++q) s += f[q];
            }
        if (kWaves > 1) __syncthreads();  // the sums are read
        join_stats<kWaves>(a.L, m, s, lds);
        base = m;
    }
    const double logp = logp_of(lab.x, base, a.L, s);
    if (tid == 0) policy_write(a, i, tk, logp);
    if (!a.grad) return;
    const float c = policy_slope(a, tk, logp), k1 = -c / s;
    if (base == -INFINITY) base = 0.0f;
    const auto write = [&](auto shift) {
        constexpr bool kShift = decltype(shift)::value;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (k * kThreads < row.nb) {
                const int j = row.head + (tid + k * kThreads) * N;
                x[k].unpack(f);
                gradient<N, kShift>(f, base, a.L, k1, c, lab.y - j);
                x[k].pack(f);
                if (tid + k * kThreads < row.nb) x[k].store_once(out + j);
            }
        if (e >= 0) {
            float g[1] = {ex};
            gradient<1, kShift>(g, base, a.L, k1, c, lab.y - e);
            out[e] = Elem<DT>::down(g[0]);
        }
    };
    if (shifted) write(std::true_type{});
    else write(std::false_type{});
}

// Rows longer than a workgroup's registers: two reads.
template <int DT>
__global__ __launch_bounds__(kRowThreads) void policy_long(PolicyArgs a) {
    typedef typename Elem<DT>::T T;
    __shared__ float2 lds[kRowThreads / 64];
    const int64_t i = row_of<kRowThreads>(), r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels[r * a.label_pitch + t];
    const int64_t at = r * a.grad_seq + t * a.grad_tok;
    T* out = static_cast<T*>(a.grad) + at;
    if (label == a.ignore) {
        policy_ignored<DT, kRowThreads>(a, i, at, threadIdx.x);
        return;
    }
    const T* in = static_cast<const T*>(a.logits) + r * a.seq + t * a.tok;
    const Label<DT> lab(in, a.V, label);
    const Token tk = policy_token(a, r, t);
    const float2 st = stream_row<DT, kRowThreads, false>({in, a.V, at}, threadIdx.x, a.L, lds);
    const double logp = logp_of(lab.x, st.x, a.L, st.y);
    if (threadIdx.x == 0) policy_write(a, i, tk, logp);
    if (!a.grad) return;
    write_gradient<DT, kRowThreads>(in, out, a.V, at, threadIdx.x, st, a.L, policy_slope(a, tk, logp), lab.y);
}

// The sum over a workgroup's threads, valid in thread 0.
template <int kWaves>
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kWaves; ++w) v += lds[w];
    __syncthreads();
    return v;
}

// The three sums over the tokens, in 64 bits and a fixed order: each workgroup a
// share, the last one to finish adds the shares.
__global__ __launch_bounds__(256) void policy_finish(PolicyArgs a) {
    __shared__ double lds[4];
    __shared__ bool last;
    double v[3] = {0.0, 0.0, 0.0};
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.rows; i += (int64_t)gridDim.x * 256) {
        const float4 k = a.tokens[i];
        v[0] += k.x;
        v[1] += k.y;
        v[2] += k.z;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) v[q] = block_sum<4>(v[q], lds);
    if (gridDim.x == 1) {
        if (threadIdx.x == 0)
            for (int q = 0; q < 3; ++q) a.stats[q] = (float)v[q];
        return;
    }
    if (threadIdx.x == 0) {
        for (int q = 0; q < 3; ++q) a.sums[q * kFinishBlocks + blockIdx.x] = v[q];
        __threadfence();
        last = atomicAdd(a.done, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last || threadIdx.x >= 3) return;
    __threadfence();
    double t = 0.0;
    for (unsigned b = 0; b < gridDim.x; ++b)
        t += __hip_atomic_load(a.sums + threadIdx.x * kFinishBlocks + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a.stats[threadIdx.x] = (float)t;
}

// -- preference -----------------------------------------------------------------

struct PrefArgs {
    const void* logits;
    void* grad;
    int64_t seq, tok, grad_seq, grad_tok;
    const int64_t* labels;
    int64_t label_pitch, ignore;
    const float* ref_logp;  // NULL: zero
    int64_t P, T;
    int32_t V;
    float beta, smoothing, scale;
    int32_t average;
    float* logp;       // [2P][T]
    float* rewards;    // [2P]
    float* pair_loss;  // [P]
    float* loss;
    int* done;         // pairs that are done
    float2* stats;     // [2P][T] (shift, sum)
    float* coef;       // [2P]
};

template <int DT, int kThreads, bool kOnce>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) void pref_logp(PrefArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int kWaves = kThreads / 64;
    __shared__ float2 lds[kWaves];
    const int tid = threadIdx.x % kThreads;
    const int64_t i = row_of<kThreads>();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;  // the next launch counts there
    if (i >= 2 * a.P * a.T) return;
    const int64_t r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels[r * a.label_pitch + t];
    if (label == a.ignore) {
        if (tid == 0) a.logp[r * a.T + t] = 0.0f;
        return;
    }
    const int64_t at = r * a.seq + t * a.tok;  // nothing is written: whole lines are read
    const T* in = static_cast<const T*>(a.logits) + at;
    const Label<DT> lab(in, a.V, label);
    const float2 st = stream_row<DT, kThreads, kOnce>({in, a.V, at}, tid, kLog2e, lds);
    if (tid == 0) {
        a.logp[r * a.T + t] = (float)logp_of(lab.x, st.x, kLog2e, st.y);
        a.stats[r * a.T + t] = st;
    }
}

// A pair's rewards, loss and both c, from its answers' sums and numbers of tokens.
struct Pair {
    double reward[2], loss, c[2];
};

__device__ __forceinline__ Pair pref_finish_pair(const PrefArgs& a, const double (&sum)[2], const int (&n)[2]) {
    Pair q;
    double share[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        share[side] = a.average ? 1.0 / (n[side] > 0 ? n[side] : 1) : 1.0;
        q.reward[side] = (double)a.beta * sum[side] * share[side];
    }
    const double h = q.reward[0] - q.reward[1], eps = a.smoothing;
    const double z = exp(-fabs(h)), low = log1p(z);  // low: -log sigmoid(|h|)
    // a side without weight is not in the sum: it is infinite where an answer is impossible
    q.loss = (eps < 1.0 ? (1.0 - eps) * (low + fmax(-h, 0.0)) : 0.0) + (eps > 0.0 ? eps * (low + fmax(h, 0.0)) : 0.0);
    // sigmoid(h) - (1 - eps) = eps sigmoid(h) - (1 - eps) sigmoid(-h)
    const double big = 1.0 / (1.0 + z), small = z / (1.0 + z);
    const double up = h >= 0.0 ? big : small, down = h >= 0.0 ? small : big;
    const double slope = (double)a.beta * (eps * up - (1.0 - eps) * down) / (double)a.P * (double)a.scale;
    q.c[0] = slope * share[0];
    q.c[1] = -slope * share[1];
    return q;
}

// What a thread adds to an answer's sum and number of tokens, `step` tokens apart.
__device__ __forceinline__ void pref_sum(const PrefArgs& a, int64_t r, int first, int step, double& sum, int& n) {
    sum = 0.0;
    n = 0;
    for (int64_t t = first; t < a.T; t += step) {
        if (a.labels[r * a.label_pitch + t] == a.ignore) continue;
        sum += (double)a.logp[r * a.T + t] - (a.ref_logp ? (double)a.ref_logp[r * a.T + t] : 0.0);
        ++n;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o);
        n += __shfl_xor(n, o);
    }
}

// A pair by one wavefront, the result in every lane.
__device__ __forceinline__ Pair pref_wave_pair(const PrefArgs& a, int64_t p) {
    double sum[2];
    int n[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) pref_sum(a, side ? a.P + p : p, threadIdx.x & 63, 64, sum[side], n[side]);
    return pref_finish_pair(a, sum, n);
}

__device__ __forceinline__ void pref_write_pair(const PrefArgs& a, int64_t p, const Pair& q) {
    a.rewards[p] = (float)q.reward[0];
    a.rewards[a.P + p] = (float)q.reward[1];
    a.pair_loss[p] = (float)q.loss;
}

// One workgroup a pair: the two implicit rewards, the loss and both c.
__global__ __launch_bounds__(256) void pref_pair(PrefArgs a) {
    __shared__ double lds[2][4];
    __shared__ int cnt[2][4];
    __shared__ bool last;
    const int64_t p = blockIdx.x;
    double sum[2];
    int n[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        pref_sum(a, side ? a.P + p : p, threadIdx.x, 256, sum[side], n[side]);
        if ((threadIdx.x & 63) == 0) {
            lds[side][threadIdx.x >> 6] = sum[side];
            cnt[side][threadIdx.x >> 6] = n[side];
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int side = 0; side < 2; ++side)
            for (int w = 1; w < 4; ++w) {
                sum[side] += lds[side][w];
                n[side] += cnt[side][w];
            }
        const Pair q = pref_finish_pair(a, sum, n);
        pref_write_pair(a, p, q);
        a.coef[p] = (float)q.c[0];
        a.coef[a.P + p] = (float)q.c[1];
    }
    // the last pair to finish takes the mean
    if (threadIdx.x == 0) {
        __threadfence();
        last = a.P == 1 || atomicAdd(a.done, 1) == (int)a.P - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < a.P; i += 256)
        v += __hip_atomic_load(a.pair_loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    v = block_sum<4>(v, lds[0]);
    if (threadIdx.x == 0) a.loss[0] = (float)(v / (double)a.P);
}
// The rows from the last to the first: of what the first launch read, the 256 MB
// cache behind the XCDs' has the last rows (16 x 512 x 50257 bf16 both launches:
// 303 us, in the first launch's order 328).  Rows of over 2048 vectors by 1024
// threads, so that few rows are under way at once (256 threads: 346 us).
//
// kPairs: few tokens; every wavefront works out its row's pair for itself, which
// spares pref_pair's launch, and the first wavefront of the launch writes the pairs.
template <int DT, int kThreads, bool kPairs>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) void pref_gradient(PrefArgs a) {
    typedef typename Elem<DT>::T T;
    const int tid = threadIdx.x % kThreads;
    const int64_t i = 2 * a.P * a.T - 1 - row_of<kThreads>();
    if (kPairs && blockIdx.x == 0 && threadIdx.x < 64) {
        double mean = 0.0;
        for (int64_t p = 0; p < a.P; ++p) {
            const Pair q = pref_wave_pair(a, p);
            mean += (float)q.loss;
            if (threadIdx.x == 0) pref_write_pair(a, p, q);
        }
        if (threadIdx.x == 0) a.loss[0] = (float)(mean / (double)a.P);
    }
    if (i < 0) return;
    const int64_t r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels[r * a.label_pitch + t];
    const int64_t at = r * a.grad_seq + t * a.grad_tok;
    T* out = static_cast<T*>(a.grad) + at;
    if (label == a.ignore) {
        zero_row<DT, kThreads>(out, a.V, at, tid);
        return;
    }
    float c;
    if constexpr (kPairs) {
        const Pair q = pref_wave_pair(a, r < a.P ? r : r - a.P);
        c = (float)(r < a.P ? q.c[0] : q.c[1]);
    } else {
        c = a.coef[r];
    }
    const int y = (uint64_t)label < (uint64_t)a.V ? (int)label : -1;
    write_gradient<DT, kThreads>(static_cast<const T*>(a.logits) + r * a.seq + t * a.tok, out, a.V, at, tid,
                                 a.stats[r * a.T + t], kLog2e, c, y);
}

// What there is without pairs, or before the first launch without tokens.
__global__ void pref_clear(float* loss, int* done) {
    if (loss) *loss = 0.0f;
    if (done) *done = 0;
}

// -- host -----------------------------------------------------------------------

// Rows of 6,657 to 13,312 vectors: by 1024 threads in 32 bits (16 x 256 tokens of 26,628
// entries 158 us, by 512 167; of 50,257 287 and 313), by 512 in 16 bits, whose rows have
// twice the elements to work on and two of which then share a CU (of 53,256 172 us, by 1024
// 191; of 65,536 212 and 215; only at the long end 1024 would gain: 106,496 336 and 328).
template <int DT>
void policy_long_rows(const PolicyArgs& a, dim3 rows, hipStream_t st) {
    if constexpr (DT == GMC_F32) policy_held<DT, 1024, 13><<<rows, 1024, 0, st>>>(a);
    else policy_held<DT, 512, 26><<<rows, 512, 0, st>>>(a);
}

constexpr int64_t kMostRows = 0xffffffffll / 1024;

bool finite_f32(double v) { return isfinite((float)v); }

// The bytes of R sequences of T rows of V elements of b bytes.
int64_t rows_span(int64_t R, int64_t T, int64_t V, int64_t seq, int64_t tok, int64_t b) {
    return ((R - 1) * (R > 1 ? seq : 0) + (T - 1) * (T > 1 ? tok : 0) + V) * b;
}

gmc_status logits_check(const char* me, int32_t dtype, int64_t R, int64_t T, int64_t V, const void* logits,
                        int64_t seq, int64_t tok, const void* grad, int64_t grad_seq, int64_t grad_tok,
                        const void* labels, int64_t label_pitch) {
    if (!known_type(dtype)) return op_error(GMC_EINVAL, me, "unknown element type");
    if (R < 0 || T < 0 || V < 1 || V > 0x3fffffff)
        return op_error(GMC_EINVAL, me, "need R >= 0, T >= 0 and 1 <= V < 2^30");
    if (R == 0 || T == 0) return GMC_OK;
    if (R > kMostRows / T) return op_error(GMC_EINVAL, me, "more than 2^22 - 1 tokens");
    if (!logits || !labels) return op_error(GMC_EINVAL, me, "NULL argument");
    const auto fits = [&](int64_t s, int64_t k) {
        constexpr int64_t kMost = int64_t(1) << 50;
        if (T > 1 && (k < V || k > kMost / T)) return false;
        return R == 1 || (s >= (T - 1) * (T > 1 ? k : 0) + V && s <= kMost / R);
    };
    if (!fits(seq, tok) || (grad && !fits(grad_seq, grad_tok)))
        return op_error(GMC_EINVAL, me, "a pitch is shorter than what it steps over");
    if (R > 1 && (label_pitch < T || label_pitch > (int64_t(1) << 50) / R))
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

using namespace gmc;

extern "C" {

int64_t gmc_policy_loss_workspace(int64_t R, int64_t T) {
    if (R < 0 || T < 0 || (T > 0 && R > kMostRows / T)) return -1;
    if (T == 0) R = 0;  // sequences without tokens, any number of them
    return R * T * (int64_t)sizeof(float4) + kFinishBlocks * 3 * (int64_t)sizeof(double) + (2 + R) * (int64_t)sizeof(float);
}

gmc_status gmc_policy_loss(void* hip_stream, int32_t dtype, int64_t R, int64_t T, int64_t V, const void* logits_dev,
                           int64_t seq_pitch, int64_t tok_pitch, const int64_t* labels_dev, int64_t label_pitch,
                           int64_t ignore, const float* old_logp_dev, const float* ref_logp_dev, const float* adv_dev,
                           int64_t adv_seq, int64_t adv_tok, double clip_lo, double clip_hi, double kl_coef,
                           double temperature, int32_t by_sequence, double grad_scale, float* stats_dev,
                           float* logp_dev, void* grad_dev, int64_t grad_seq, int64_t grad_tok, void* workspace_dev,
                           int64_t workspace_bytes) {
    const char* me = "gmc_policy_loss";
    const gmc_status ok = logits_check(me, dtype, R, T, V, logits_dev, seq_pitch, tok_pitch, grad_dev, grad_seq,
                                       grad_tok, labels_dev, label_pitch);
    if (ok != GMC_OK) return ok;
    if (!(clip_lo >= 0.0 && clip_lo <= 1.0 && clip_hi >= 0.0 && isfinite(clip_hi)))
        return op_error(GMC_EINVAL, me, "need 0 <= clip_lo <= 1 and 0 <= clip_hi");
    if (!finite_f32(kl_coef) || !finite_f32(grad_scale))
        return op_error(GMC_EINVAL, me, "kl_coef and grad_scale must be finite in fp32");
    if (!(temperature > 0.0 && isfinite(temperature) && finite_f32(1.4426950408889634 / temperature)))
        return op_error(GMC_EINVAL, me, "temperature must be > 0 and finite, log2(e) / temperature finite in fp32");
    if (!stats_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    if (workspace_bytes < gmc_policy_loss_workspace(R, T) || !workspace_dev)
        return op_error(GMC_EINVAL, me, "the workspace is too small");
    if (reinterpret_cast<uintptr_t>(workspace_dev) & 15u)
        return op_error(GMC_EINVAL, me, "the workspace is not 16-byte aligned");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    PolicyArgs a{};
    a.rows = R * T;
    a.tokens = static_cast<float4*>(workspace_dev);
    if (a.rows) {
        if (!adv_dev || !logp_dev) return op_error(GMC_EINVAL, me, "NULL argument");
        constexpr int64_t kFar = int64_t(1) << 50;
        const auto reach = [](int64_t steps, int64_t pitch) { return steps > 0 ? steps * pitch : 0; };
        if ((R > 1 && (adv_seq < -kFar / R || adv_seq > kFar / R)) || (T > 1 && (adv_tok < -kFar / T || adv_tok > kFar / T)))
            return op_error(GMC_EINVAL, me, "a pitch of the advantages is out of range");
        const int64_t by_seq = reach(R - 1, adv_seq), by_tok = reach(T - 1, adv_tok);
        const int64_t below = (by_seq < 0 ? by_seq : 0) + (by_tok < 0 ? by_tok : 0);
        const int64_t above = (by_seq > 0 ? by_seq : 0) + (by_tok > 0 ? by_tok : 0);
        const int64_t b = type_size(dtype), n = a.rows * 4;
        const Span stats(stats_dev, 12), logp(logp_dev, n), scratch(workspace_dev, gmc_policy_loss_workspace(R, T));
        if (!apart({stats, logp, scratch, {grad_dev, rows_span(R, T, V, grad_seq, grad_tok, b)}},
                   {{labels_dev, rows_span(R, 1, T, label_pitch, 0, 8)}, {old_logp_dev, n}, {ref_logp_dev, n},
                    {adv_dev + below, (above - below + 1) * 4}}) ||
            !apart({stats, logp, scratch}, {{logits_dev, rows_span(R, T, V, seq_pitch, tok_pitch, b)}}))
            return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
        a.sums = reinterpret_cast<double*>(a.tokens + a.rows);
        a.done = reinterpret_cast<int*>(a.sums + 3 * kFinishBlocks);
        float* weight = reinterpret_cast<float*>(a.done + 1);
        a.logits = logits_dev;
        a.grad = grad_dev;
        a.seq = seq_pitch;
        a.tok = tok_pitch;
        // without a gradient, the order of one with the pitches given or of a contiguous one
        a.grad_seq = grad_dev || grad_tok > 0 ? grad_seq : T * V;
        a.grad_tok = grad_dev || grad_tok > 0 ? grad_tok : V;
        a.labels = labels_dev;
        a.label_pitch = label_pitch;
        a.ignore = ignore;
        a.old_logp = old_logp_dev;
        a.ref_logp = ref_logp_dev;
        a.adv = adv_dev;
        a.adv_seq = adv_seq;
        a.adv_tok = adv_tok;
        a.R = R;
        a.T = T;
        a.V = (int32_t)V;
        a.lo = (float)clip_lo;
        a.hi = (float)clip_hi;
        a.kl = (float)kl_coef;
        a.L = (float)(1.4426950408889634 / temperature);
        a.inv_tau = (float)(1.0 / temperature);
        a.scale = (float)grad_scale;
        a.by_sequence = by_sequence != 0;
        a.logp = logp_dev;
        a.weight = weight;
        const int64_t vecs = V * type_size(dtype) / 16;  // at most, whatever the alignment
        const bool held = vecs <= 1024 * kLongest;
        if (held && !a.by_sequence && a.rows <= kRowTokens) {
            a.weight = nullptr;
        } else if (a.rows > kFewTokens || R > kFewSequences) {
            policy_counts<<<dim3((unsigned)((R + 3) / 4)), 256, 0, st>>>(a, weight);
            policy_weight<true><<<1, 1024, 0, st>>>(a, weight);
        } else {
            policy_weight<false><<<1, 1024, 0, st>>>(a, weight);
        }
        const dim3 rows((unsigned)a.rows), quads((unsigned)((a.rows + 3) / 4));
        GMC_BY_TYPE(dtype, {
            if (vecs <= 64 * 8) policy_held<DT, 64, 8><<<quads, 256, 0, st>>>(a);
            else if (vecs <= 256 * 8) policy_held<DT, 256, 8><<<rows, 256, 0, st>>>(a);
            else if (vecs <= 512 * 8) policy_held<DT, 512, 8><<<rows, 512, 0, st>>>(a);
            else if (vecs <= 512 * 13) policy_held<DT, 512, 13><<<rows, 512, 0, st>>>(a);
            else if (vecs <= 512 * 26) policy_long_rows<DT>(a, rows, st);
            else if (held) policy_held<DT, 1024, kLongest><<<rows, 1024, 0, st>>>(a);
            else policy_long<DT><<<rows, kRowThreads, 0, st>>>(a);
        });
    }
    a.stats = stats_dev;
    const int64_t shares = (a.rows + 1023) / 1024;
    const unsigned finish = a.rows <= 2 * kRowTokens ? 1u : shares > kFinishBlocks ? (unsigned)kFinishBlocks : (unsigned)shares;
    policy_finish<<<dim3(finish), 256, 0, st>>>(a);
    return op_launched(me);
}

int64_t gmc_preference_loss_workspace(int64_t P, int64_t T) {
    if (P < 0 || P > kMostRows / 2 || T < 0 || (T > 0 && P > kMostRows / 2 / T)) return -1;
    return 2 * P * T * (int64_t)sizeof(float2) + (2 * P + 2) * (int64_t)sizeof(float);
}

gmc_status gmc_preference_loss(void* hip_stream, int32_t dtype, int64_t P, int64_t T, int64_t V,
                               const void* logits_dev, int64_t seq_pitch, int64_t tok_pitch, const int64_t* labels_dev,
                               int64_t label_pitch, int64_t ignore, const float* ref_logp_dev, double beta,
                               double smoothing, int32_t average, double grad_scale, float* loss_dev,
                               float* pair_loss_dev, float* rewards_dev, float* logp_dev, void* grad_dev,
                               int64_t grad_seq, int64_t grad_tok, void* workspace_dev, int64_t workspace_bytes) {
    const char* me = "gmc_preference_loss";
    if (P < 0 || P > kMostRows / 2) return op_error(GMC_EINVAL, me, "need 0 <= P < 2^21");
    const gmc_status ok = logits_check(me, dtype, 2 * P, T, V, logits_dev, seq_pitch, tok_pitch, grad_dev, grad_seq,
                                       grad_tok, labels_dev, label_pitch);
    if (ok != GMC_OK) return ok;
    if (!finite_f32(beta) || !finite_f32(grad_scale))
        return op_error(GMC_EINVAL, me, "beta and grad_scale must be finite in fp32");
    if (!(smoothing >= 0.0 && smoothing <= 1.0)) return op_error(GMC_EINVAL, me, "smoothing must be in [0, 1]");
    if (!loss_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (P > 0) {
        if (!pair_loss_dev || !rewards_dev || (T > 0 && !logp_dev)) return op_error(GMC_EINVAL, me, "NULL argument");
        if (!workspace_dev || workspace_bytes < gmc_preference_loss_workspace(P, T))
            return op_error(GMC_EINVAL, me, "the workspace is too small");
        if (reinterpret_cast<uintptr_t>(workspace_dev) & 7u)
            return op_error(GMC_EINVAL, me, "the workspace is not 8-byte aligned");
        const int64_t R = 2 * P, b = type_size(dtype), some = T > 0;
        const Span loss(loss_dev, 4), each(pair_loss_dev, P * 4), rewards(rewards_dev, R * 4), logp(logp_dev, R * T * 4),
            scratch(workspace_dev, gmc_preference_loss_workspace(P, T));
        if (!apart({loss, each, rewards, logp, scratch, {grad_dev, some * rows_span(R, T, V, grad_seq, grad_tok, b)}},
                   {{labels_dev, some * rows_span(R, 1, T, label_pitch, 0, 8)}, {ref_logp_dev, R * T * 4}}) ||
            !apart({loss, each, rewards, logp, scratch}, {{logits_dev, some * rows_span(R, T, V, seq_pitch, tok_pitch, b)}}))
            return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
        PrefArgs a{};
        a.logits = logits_dev;
        a.grad = grad_dev;
        a.seq = seq_pitch;
        a.tok = tok_pitch;
        a.grad_seq = grad_seq;
        a.grad_tok = grad_tok;
        a.labels = labels_dev;
        a.label_pitch = label_pitch;
        a.ignore = ignore;
        a.ref_logp = ref_logp_dev;
        a.P = P;
        a.T = T;
        a.V = (int32_t)V;
        a.beta = (float)beta;
        a.smoothing = (float)smoothing;
        a.scale = (float)grad_scale;
        a.average = average != 0;
        a.logp = logp_dev;
        a.rewards = rewards_dev;
        a.pair_loss = pair_loss_dev;
        a.stats = static_cast<float2*>(workspace_dev);
        a.coef = reinterpret_cast<float*>(a.stats + 2 * P * T);
        a.done = reinterpret_cast<int*>(a.coef + 2 * P);
        a.loss = loss_dev;
        const int64_t tokens = 2 * P * T, vecs = V * type_size(dtype) / 16;
        const dim3 rows((unsigned)tokens), quads((unsigned)((tokens + 3) / 4));
        GMC_BY_TYPE(dtype, {
            if (tokens) {
                if (vecs <= 64 * 8) pref_logp<DT, 64, false><<<quads, 256, 0, st>>>(a);
                else if (a.grad) pref_logp<DT, kStatThreads, false><<<rows, kStatThreads, 0, st>>>(a);
                else pref_logp<DT, kStatThreads, true><<<rows, kStatThreads, 0, st>>>(a);
            } else {
                pref_clear<<<1, 1, 0, st>>>(nullptr, a.done);
            }
            const bool few = a.grad && tokens && P <= kRowPairs && P * T <= kRowPairTokens;
            if (!few) pref_pair<<<dim3((unsigned)P), 256, 0, st>>>(a);
            if (tokens && a.grad) {
                if (vecs <= 64 * 8) {
                    if (few) pref_gradient<DT, 64, true><<<quads, 256, 0, st>>>(a);
                    else pref_gradient<DT, 64, false><<<quads, 256, 0, st>>>(a);
                } else {
                    if (few) pref_gradient<DT, kStatThreads, true><<<rows, kStatThreads, 0, st>>>(a);
                    else if (vecs <= 2048) pref_gradient<DT, 512, false><<<rows, 512, 0, st>>>(a);
                    else pref_gradient<DT, 1024, false><<<rows, 1024, 0, st>>>(a);
                }
            }
        });
    } else {
        pref_clear<<<1, 1, 0, st>>>(loss_dev, nullptr);
    }
    return op_launched(me);
}

}  // extern "C"
