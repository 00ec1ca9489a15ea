// The scores of tokens from their logits (gmc_token_scores in include/gmc.h: the
// log-probabilities of given tokens, entropies and the most probable tokens) and the
// logits' gradient from the scores' (gmc_token_scores_backward).
//
// With e_j = 2^t_j, t_j = (x_j - max) L, L = log2(e) / tau, one row needs
//   max,  S = sum e_j,  U = sum e_j t_j:
//   log p_y = (x_y - max) / tau - ln S,  H = ln S - ln 2 U / S.
// A row is read once and held in registers, so that the maximum is known before
// the exponentials: every t_j is <= 0, no sum overflows, and neither ln S nor U / S
// cancels.  Entries of -inf have e_j = 0 and t_j no smaller than -160, so that
// e_j t_j is 0 too.
//
// The `top` largest: entries are ordered by a 64-bit key, the value's ordered bits
// above the complement of its place, so no two are equal and ties go to the lower
// place.  Each wavefront finds its ceil(top / wavefronts)-th largest of its threads'
// maxima; the least of these is a threshold that at least `top` entries reach and few
// more; they are collected in shared memory and each counts the keys above it.
// Where too many reach it (equal logits, few that are not -inf) and in rows with a
// NaN the largest key below the last one is taken, `top` times.
//
// Rows beyond a workgroup's registers, and rows of a call with few of them, are cut
// into pieces, each with its own maximum, sums and largest keys, which a second launch
// joins.
//
// What bounds it.  Batches are memory's: 16 x 1024 x 50257 bf16, 9941 tokens counting, 170 to 194 us (5.9 to 5.2 TB/s),
// the gradient of half as many 237 (5.6, reads and writes).  16-bit rows with alternatives and lengths that no line
// divides: the exponentials and each row's chain (6 x 333 x 32003 f16, 8 of them: 13 us of 21).  Few rows: one row's
// chain of load, maximum, sums and choice (one 9 us, 20 alternatives of 64 rows 13.5).
#include "gmc_rows.h"

namespace gmc {

namespace {

constexpr int kMostTop = 32;
constexpr int kMostKeys = 1024;      // a row's (or piece's) entries that reach the threshold
constexpr int kRowKeys = 256;        // of a row by one wavefront
constexpr int kJoinKeys = 1024;      // keys the joining launch looks at at once
constexpr float kNoShare = -160.0f;  // 2^-160 is 0 in 32 bits

struct ScoreArgs {
    const void* logits;
    int64_t seq, tok;
    const int64_t* labels;  // NULL: none
    int64_t label_pitch, ignore;
    int64_t T, rows;
    int32_t V, piece, pieces, top;
    float L, inv_tau;
    float *logp, *entropy, *top_logp, *norm;
    int64_t* top_ids;
    float4* part;    // per piece: maximum, S, U
    uint64_t* keys;  // per piece: its `top` largest
};

// NaN where one of the two is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A NaN is above +inf (0xff800000) and below what no key is: ~0, with which a search for the largest key
// begins, would be its own at place 0.
constexpr uint32_t kNanOrder = 0xfffffffeu;

__device__ __forceinline__ uint64_t key_of(float x, int j) {
    const uint32_t b = __float_as_uint(x + 0.0f);   // -0 as 0
    const uint32_t o = x != x ? kNanOrder : b >> 31 ? ~b : b | 0x80000000u;
    return (uint64_t)o << 32 | (uint32_t)~j;
}
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return o == kNanOrder ? NAN : __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_place(uint64_t k) { return (int)~(uint32_t)k; }

// A value of the lane that a fixed pattern pairs with this one.
template <int kPattern>
__device__ __forceinline__ float paired(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kPattern, 15, 15, true));
}
__device__ __forceinline__ float of_lane(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
// The wavefront's values joined, in every lane: within 16 lanes by patterns (neighbours, pairs, halves and
// rows mirrored), then the four rows' by reading a lane of each.  An exchange by address takes 15
// times as long as a pattern, and a row's six such joins would be most of a short row's time.
template <class F>
__device__ __forceinline__ float wave_join(float v, F&& op) {
    v = op(v, paired<0xb1>(v));
    v = op(v, paired<0x4e>(v));
    v = op(v, paired<0x141>(v));
    v = op(v, paired<0x140>(v));
    return op(op(of_lane(v, 0), of_lane(v, 16)), op(of_lane(v, 32), of_lane(v, 48)));
}
__device__ __forceinline__ float lanes_sum(float v) {
    return wave_join(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float lanes_max(float v) {
    return wave_join(v, [](float a, float b) { return larger(a, b); });
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t w = __shfl_xor(v, o);
        v = w > v ? w : v;
    }
    return v;
}

// What the threads of a row share, a row being kWaves wavefronts': all of a workgroup's
// (then their barrier is the workgroup's) or one.
template <int kWaves>
__device__ __forceinline__ void row_barrier() {
    if constexpr (kWaves > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int kWaves>
struct Shared {
    static constexpr int kKeys = kWaves == 1 ? kRowKeys : kMostKeys, kVectors = kKeys / 4;
    float top[kWaves];
    float2 sum[kWaves];
    float reach[kWaves];
    uint64_t best[2][kWaves];
    int count, vectors;
    uint64_t keys[kKeys];
    uint4 vector[kVectors];   // with an entry that reaches the threshold
    int place[kVectors];      // of its first entry
};

__device__ __forceinline__ float log_sum(float m, float s) { return fabsf(m) < INFINITY ? logf(s) : NAN; }

// A logit's distance to the maximum over the temperature; -inf stays, also where 1 / tau is 0 in 32 bits.
__device__ __forceinline__ float scaled(const ScoreArgs& a, float x, float m) { return x == -INFINITY ? x : (x - m) * a.inv_tau; }

__device__ __forceinline__ void write_scores(const ScoreArgs& a, int64_t i, float m, float s, float u, float xy) {
    const float ls = log_sum(m, s);
    reinterpret_cast<float2*>(a.norm)[i] = make_float2(m, ls);
    a.entropy[i] = ls - 0.69314718055994531f * (u / s);
    if (a.logp) a.logp[i] = scaled(a, xy, m) - ls;
}

__device__ __forceinline__ void write_top(const ScoreArgs& a, int64_t i, int rank, uint64_t key, float m, float s) {
    a.top_ids[i * a.top + rank] = key_place(key);
    a.top_logp[i * a.top + rank] = scaled(a, key_value(key), m) - log_sum(m, s);
}

// The scores of a token that is ignored.
__device__ __forceinline__ void write_ignored(const ScoreArgs& a, int64_t i, int tid) {
    if (tid == 0) {
        reinterpret_cast<float2*>(a.norm)[i] = make_float2(0.0f, 0.0f);
        a.entropy[i] = 0.0f;
        a.logp[i] = 0.0f;
    }
    if (tid < a.top) {
        a.top_ids[i * a.top + tid] = -1;
        a.top_logp[i * a.top + tid] = 0.0f;
    }
}

template <int DT>
__device__ __forceinline__ float label_logit(const typename Elem<DT>::T* row, int V, int64_t label) {
    return (uint64_t)label < (uint64_t)V ? Elem<DT>::up(row[label]) : NAN;
}

// The row, or piece of one, of a workgroup, or of a wavefront where four share one, in the launch's
// order, which deals the tokens of a sequence out to all XCDs: where many of a run of rows are ignored, a
// run for each XCD leaves some with little to do (6 x 333 x 32003 f16, three fifths of the tokens counting:
// 29 us, dealt out 22; 16 x 1024 x 50257 bf16 180 us and 170).
template <int kThreads>
__device__ __forceinline__ int64_t in_turn() {
    if constexpr (kThreads == 64) return (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    else return blockIdx.x;
}

// Vectors that are looked at another time are unpacked another time: kept unpacked, 16-bit
// ones would take twice their registers.
template <int DT, int N, int kHeld>
__device__ __forceinline__ void again(Vec<DT, N> (&x)[kHeld]) {
    if constexpr (DT != GMC_F32)
#pragma unroll
        for (int k = 0; k < kHeld; ++k) asm volatile("" : "+v"(x[k].raw));
}

// One row, or a piece of one (kPieces), per kThreads threads, held in kHeld vectors a
// thread.
template <int DT, int kThreads, int kHeld, bool kTop, bool kPieces>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) __attribute__((amdgpu_waves_per_eu(kHeld <= 8 ? 6 : 4)))
void score_rows(ScoreArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int N = 16 / Elem<DT>::kSize;
    constexpr int kWaves = kThreads / 64;
    typedef Vec<DT, N> V;
    __shared__ Shared<kWaves> shared[kThreads == 64 ? 4 : 1];
    Shared<kWaves>& sh = shared[kThreads == 64 ? threadIdx.x >> 6 : 0];
    const int tid = threadIdx.x % kThreads, wave = tid >> 6, lane = tid & 63;
    const int64_t id = in_turn<kThreads>();
    const int64_t i = kPieces ? id / a.pieces : id;
    if (i >= a.rows) return;
    const int from = kPieces ? (int)(id - i * a.pieces) * a.piece : 0;
    const int len = kPieces && a.V - from > a.piece ? a.piece : a.V - from;
    const int64_t r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels ? a.labels[r * a.label_pitch + t] : 0;
    if (a.labels && label == a.ignore) {
        if (!kPieces) write_ignored(a, i, tid);
        return;
    }
    const int64_t at = r * a.seq + t * a.tok;
    const T* in = static_cast<const T*>(a.logits) + at;
    const Row<DT, kThreads> row(in + from, len, at + from);
    // past the end a vector holds -inf
    V x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        x[k] = nothing<DT, N>();
        if (tid + k * kThreads < row.nb) x[k] = V::load_once(row.p + row.head + (int64_t)(tid + k * kThreads) * N);
    }
    const int e = row.edge(tid);
    const float ex = e >= 0 ? Elem<DT>::up(row.p[e]) : -INFINITY;
    float xy = NAN;
    if (!kPieces && a.labels && tid == 0) xy = label_logit<DT>(in, a.V, label);
    float f[N], own = ex;
    if constexpr (DT == GMC_F16) {
        // two at a time, as they are: unpacked, the largest takes three times as many operations
        typedef _Float16 Pair __attribute__((ext_vector_type(2)));
        struct Pairs {
            Pair p[N / 2];
        };
        Pair most = {(_Float16)-INFINITY, (_Float16)-INFINITY};
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (k * kThreads < row.nb) {
                const Pairs h = __builtin_bit_cast(Pairs, x[k].raw);
#pragma unroll
                for (int q = 0; q < N / 2; ++q) most = __builtin_elementwise_maximum(most, h.p[q]);
            }
        own = larger(own, larger((float)most.x, (float)most.y));
    } else {
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (k * kThreads < row.nb) {
                x[k].unpack(f);
#pragma unroll
                for (int q = 0; q < N; ++q) own = larger(own, f[q]);
            }
    }
    float m = lanes_max(own);
    if constexpr (kWaves > 1) {
        if (lane == 0) sh.top[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = larger(m, sh.top[w]);
    }
    const float base = m == -INFINITY ? 0.0f : m;
    const float ve = fmaxf((ex - base) * a.L, kNoShare);
    float s = exp2_fast(ve), u = s * ve;
    again(x);
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (k * kThreads < row.nb) {
            x[k].unpack(f);
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float v = fmaxf((f[q] - base) * a.L, kNoShare), w = exp2_fast(v);
                s += w;
                u = __builtin_fmaf(w, v, u);
            }
        }
    s = lanes_sum(s);
    u = lanes_sum(u);
    if constexpr (kTop) {
        // the wavefront's share of the threshold: its n-th largest of the threads' maxima
        float left = own != own ? INFINITY : own, least = -INFINITY;
        for (int n = (a.top + kWaves - 1) / kWaves; n > 0; --n) {
            least = lanes_max(left);
            const uint64_t who = __ballot(left == least);
            if (lane == __ffsll((unsigned long long)who) - 1) left = -INFINITY;
        }
        if (lane == 0) sh.reach[wave] = least;
        if (tid == 0) sh.count = sh.vectors = 0;
    }
    if (kWaves > 1 && lane == 0) sh.sum[wave] = make_float2(s, u);
    row_barrier<kWaves>();
    if constexpr (kWaves > 1) {
        s = u = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            s += sh.sum[w].x;
            u += sh.sum[w].y;
        }
    }
    if (tid == 0) {
        if constexpr (kPieces) a.part[id] = make_float4(m, s, u, 0.0f);
        else write_scores(a, i, m, s, u, xy);
    }
    if constexpr (kTop) {
        float reach = sh.reach[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) reach = fminf(reach, sh.reach[w]);
        typedef Shared<kWaves> S;
        const auto take = [&](float v, int j) {
            if (v >= reach) {
                const int n = atomicAdd(&sh.count, 1);
                if (n < S::kKeys) sh.keys[n] = key_of(v, from + j);
            }
        };
        // the vectors with such an entry go to shared memory whole, and their entries are looked at from
        // there, one a thread
        again(x);
        if (own >= reach) {
            if (e >= 0) take(ex, e);
#pragma unroll
            for (int k = 0; k < kHeld; ++k)
                if (tid + k * kThreads < row.nb) {
                    x[k].unpack(f);
                    float most = f[0];
#pragma unroll
                    for (int q = 1; q < N; ++q) most = fmaxf(most, f[q]);
                    if (most >= reach) {
                        const int n = atomicAdd(&sh.vectors, 1);
                        if (n < S::kVectors) {
                            sh.vector[n] = __builtin_bit_cast(uint4, x[k].raw);
                            sh.place[n] = row.head + (tid + k * kThreads) * N;
                        }
                    }
                }
        }
        row_barrier<kWaves>();
        const int vectors = sh.vectors;
        if (vectors <= S::kVectors)
            for (int c = tid; c < vectors * N; c += kThreads)
                take(Elem<DT>::up(reinterpret_cast<const T*>(sh.vector)[c]), sh.place[c / N] + c % N);
        row_barrier<kWaves>();
        const int n = sh.count, all = len < a.top ? len : a.top;
        const auto give = [&](int rank, uint64_t key) {
            if constexpr (kPieces) a.keys[id * a.top + rank] = key;
            else write_top(a, i, rank, key, m, s);
        };
        if (m == m && vectors <= S::kVectors && n <= S::kKeys) {
            for (int c = tid; c < n; c += kThreads) {
                const uint64_t key = sh.keys[c];
                int rank = 0;
#pragma unroll 8
                for (int o = 0; o < n; ++o) rank += sh.keys[o] > key;
                if (rank < all) give(rank, key);
            }
        } else {
            uint64_t last = ~uint64_t(0), best = last;
            for (int rank = 0; rank < all; ++rank) {
                if (best >= last) {
                    // read again: such rows are few, and their code would take the others' registers
                    best = 0;
                    const auto look = [&](float v, int j) {
                        const uint64_t key = key_of(v, from + j);
                        if (key < last && key > best) best = key;
                    };
                    if (e >= 0) look(ex, e);
#pragma unroll 1
                    for (int v = tid; v < row.nb; v += kThreads) {
                        V::load(row.p + row.head + (int64_t)v * N).unpack(f);
#pragma unroll
                        for (int q = 0; q < N; ++q) look(f[q], row.head + v * N + q);
                    }
                }
                uint64_t top = wave_max(best);
                if constexpr (kWaves > 1) {
                    if (lane == 0) sh.best[rank & 1][wave] = top;
                    __syncthreads();
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) top = sh.best[rank & 1][w] > top ? sh.best[rank & 1][w] : top;
                }
                if (tid == 0) give(rank, top);
                last = top;
            }
        }
        if (kPieces && tid >= all && tid < a.top) a.keys[id * a.top + tid] = 0;   // below every key
    }
}

// A row's pieces joined, by one workgroup.
template <int DT>
__global__ __launch_bounds__(256) void score_join(ScoreArgs a) {
    __shared__ float lds[4];
    __shared__ float2 sums[4];
    __shared__ uint64_t keys[kJoinKeys], kept[kMostTop];
    __shared__ int count;
    const int64_t i = blockIdx.x, r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels ? a.labels[r * a.label_pitch + t] : 0;
    if (a.labels && label == a.ignore) {
        write_ignored(a, i, threadIdx.x);
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const float4* part = a.part + i * a.pieces;
    float m = -INFINITY;
    for (int p = threadIdx.x; p < a.pieces; p += 256) m = larger(m, part[p].x);
    m = lanes_max(m);
    if (lane == 0) lds[wave] = m;
    __syncthreads();
    m = larger(larger(lds[0], lds[1]), larger(lds[2], lds[3]));
    const float base = m == -INFINITY ? 0.0f : m;
    float s = 0.0f, u = 0.0f;
    for (int p = threadIdx.x; p < a.pieces; p += 256) {
        const float4 v = part[p];
        const float d = fmaxf((v.x - base) * a.L, kNoShare), w = exp2_fast(d);
        s += w * v.y;
        u += w * __builtin_fmaf(d, v.y, v.z);
    }
    s = lanes_sum(s);
    u = lanes_sum(u);
    if (lane == 0) sums[wave] = make_float2(s, u);
    __syncthreads();
    s = sums[0].x + sums[1].x + sums[2].x + sums[3].x;
    u = sums[0].y + sums[1].y + sums[2].y + sums[3].y;
    if (threadIdx.x == 0) {
        float xy = NAN;
        if (a.labels) xy = label_logit<DT>(static_cast<const typename Elem<DT>::T*>(a.logits) + r * a.seq + t * a.tok, a.V, label);
        write_scores(a, i, m, s, u, xy);
    }
    if (!a.top) return;
    // A piece's last key has `top` at or above it: of all keys those below the greatest of these are left out.
    const uint64_t* from = a.keys + i * a.pieces * a.top;
    uint64_t least = 0;
    for (int p = threadIdx.x; p < a.pieces; p += 256) {
        const uint64_t key = from[(int64_t)p * a.top + a.top - 1];
        least = key > least ? key : least;
    }
    least = wave_max(least);
    if (lane == 0) keys[wave] = least;
    if (threadIdx.x < kMostTop) kept[threadIdx.x] = 0;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) least = keys[w] > least ? keys[w] : least;
    // the largest so far and as many others as fit beside them, until all have been looked at
    const int64_t all = (int64_t)a.pieces * a.top;
    int have = 0;
    for (int64_t done = 0; done < all;) {
        const int fit = kJoinKeys - have, n = (int)(all - done < fit ? all - done : fit);
        __syncthreads();
        for (int c = threadIdx.x; c < have + n; c += 256) {
            const uint64_t key = c < have ? kept[c] : from[done + c - have];
            if (key && key >= least) keys[atomicAdd(&count, 1)] = key;
        }
        __syncthreads();
        const int some = count;
        for (int c = threadIdx.x; c < some; c += 256) {
            const uint64_t key = keys[c];
            int rank = 0;
#pragma unroll 8
            for (int o = 0; o < some; ++o) rank += keys[o] > key;
            if (rank < a.top) kept[rank] = key;
        }
        __syncthreads();
        if (threadIdx.x == 0) count = 0;
        have = some < a.top ? some : a.top;
        done += n;
    }
    if ((int)threadIdx.x < a.top) write_top(a, i, threadIdx.x, kept[threadIdx.x], m, s);
}

// -- the gradient -------------------------------------------------------------------

struct SlopeArgs {
    const void* logits;
    void* grad;
    int64_t seq, tok, grad_seq, grad_tok;
    const int64_t* labels;
    int64_t label_pitch, ignore;
    int64_t T, rows;
    int32_t V, piece, pieces, top;
    float L, inv_tau;
    const float *norm, *entropy, *dlogp, *dentropy, *dtop;
    const int64_t* top_ids;
};

// With q_j = log2 p_j:  grad_j = p_j (c + d q_j) + what its own log-probability gets,
//   c = -(dlogp + sum dtop + dentropy H) / tau,  d = -dentropy ln 2 / tau.
// The few entries with something of their own are written again after the row (their
// logits are read before it).
template <int DT, int kThreads>
__global__ __launch_bounds__(kThreads == 64 ? 256 : kThreads) void score_gradient(SlopeArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int N = 16 / Elem<DT>::kSize;
    constexpr int kWaves = kThreads / 64;
    constexpr int kBatch = 4;
    typedef Vec<DT, N> V;
    __shared__ int64_t places[kThreads == 64 ? 4 : 1][kMostTop + 1];
    __shared__ float gains[kThreads == 64 ? 4 : 1][kMostTop + 1];
    int64_t* place = places[kThreads == 64 ? threadIdx.x >> 6 : 0];
    float* gain = gains[kThreads == 64 ? threadIdx.x >> 6 : 0];
    const int tid = threadIdx.x % kThreads;
    const int64_t id = row_of<kThreads>(), i = id / a.pieces;
    if (i >= a.rows) return;
    const int from = (int)(id - i * a.pieces) * a.piece;
    const int len = a.V - from > a.piece ? a.piece : a.V - from;
    const int64_t r = i / a.T, t = i - r * a.T;
    const int64_t label = a.labels ? a.labels[r * a.label_pitch + t] : 0;
    const int64_t at = r * a.grad_seq + t * a.grad_tok + from;
    T* out = static_cast<T*>(a.grad) + at;
    if (a.labels && label == a.ignore) {
        zero_row<DT, kThreads>(out, len, at, tid);
        return;
    }
    const float2 norm = reinterpret_cast<const float2*>(a.norm)[i];
    const float dh = a.dentropy ? a.dentropy[i] : 0.0f, H = a.dentropy ? a.entropy[i] : 0.0f;
    const float own = a.dlogp && a.labels ? a.dlogp[i] : 0.0f;
    const bool known = (uint64_t)label < (uint64_t)a.V;
    float all = own;
    for (int k = 0; k < a.top; ++k) {
        const int64_t j = a.top_ids[i * a.top + k];
        const float g = a.dtop[i * a.top + k];
        if ((uint64_t)j < (uint64_t)a.V) all += g;
    }
    if (a.dlogp && a.labels && !known) all = NAN;
    const float shift = -norm.y * kLog2e;
    float c = -(all + dh * H) * a.inv_tau;
    const float d = -dh * 0.69314718055994531f * a.inv_tau;
    if (!(fabsf(norm.x) < INFINITY) || norm.y != norm.y) c = NAN;
    const auto slope = [&](float x) {
        const float q = fmaxf(__builtin_fmaf(x - norm.x, a.L, shift), kNoShare);
        return exp2_fast(q) * __builtin_fmaf(d, q, c);
    };
    const T* in = static_cast<const T*>(a.logits) + r * a.seq + t * a.tok + from;
    float special = 0.0f;
    int64_t mine = -1;
    if (tid <= a.top) {
        const bool first = tid == a.top;   // the label stands behind the others
        const int64_t j = first ? (a.dlogp && a.labels ? label : -1) : a.top_ids[i * a.top + tid];
        place[tid] = j;
        gain[tid] = first ? own : a.dtop[i * a.top + tid];
        if ((uint64_t)j < (uint64_t)a.V && j >= from && j < from + len) {
            mine = j - from;
            special = Elem<DT>::up(in[mine]);
        }
    }
    if constexpr (kWaves > 1) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"), __builtin_amdgcn_wave_barrier();
    const Row<DT, kThreads> row(in, len, at);
    for (int v0 = tid; v0 < row.nb; v0 += kBatch * kThreads) {
        V x[kBatch];
        float f[N];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (v0 + k * kThreads < row.nb) x[k] = V::load_once(row.p + row.head + (int64_t)(v0 + k * kThreads) * N);
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (v0 + k * kThreads < row.nb) {
                x[k].unpack(f);
#pragma unroll
                for (int q = 0; q < N; ++q) f[q] = slope(f[q]);
                x[k].pack(f);
                x[k].store_once(out + row.head + (int64_t)(v0 + k * kThreads) * N);
            }
    }
    const int e = row.edge(tid);
    if (e >= 0) out[e] = Elem<DT>::down(slope(Elem<DT>::up(row.p[e])));
    if constexpr (kWaves > 1) {
        __syncthreads();   // the row is written
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        __builtin_amdgcn_wave_barrier();
    }
    if (mine < 0) return;
    float sum = 0.0f;
    for (int k = a.top; k >= 0; --k) {
        if (place[k] != mine + from) continue;
        if (k > tid) return;   // the last of the same writes
        sum += gain[k];
    }
    out[mine] = Elem<DT>::down(__builtin_fmaf(sum, a.inv_tau, slope(special)));
}

// -- host -----------------------------------------------------------------------------

// How a call's rows are cut.  Held: up to 8 vectors by each of 64 (four rows a workgroup), 256 or 512
// threads, or 13 by 512 or 1024.
struct Cut {
    int threads, held, pieces;
    int32_t piece;
};

constexpr int64_t kPlaces = 256;       // CUs
constexpr int64_t kHeldLines = 512 * 13 * 16 / 128;  // of a piece: two such workgroups share a CU
constexpr int64_t kShortPiece = 2048;  // vectors: of a row of a call with few

Cut held_by(int64_t vecs, int pieces, int32_t piece) {
    return {vecs <= 64 * 8 ? 64 : vecs <= 256 * 8 ? 256 : vecs <= 512 * 13 ? 512 : 1024, vecs <= 512 * 8 ? 8 : 13, pieces, piece};
}

// `pieces` of whole lines, so that every piece begins where the row's own lines do.
Cut in_pieces(int64_t V, int64_t b, int64_t pieces) {
    const int64_t lines = (V * b + 127) / 128, each = (lines + pieces - 1) / pieces;
    const int32_t piece = (int32_t)(each * (128 / b));
    Cut c = held_by(each * 8, (int)((V + piece - 1) / piece), piece);
    if (c.threads == 64) c.threads = 256;
    return c;
}

// Rows too long to hold are cut, into more pieces where they leave CUs without one.  Rows of 6657 to 13,312 vectors are
// held by 1024 threads, of which a CU takes one row at a time: with few rows that spares a launch (f32 x 50257, 64 rows
// 12.6 us, in pieces 15; 256 rows 11.4 and 15), with many the loads of one do not overlap the sums of another, and pieces
// of 512 threads, two on a CU, would be faster (4096 rows 150 us, in pieces 126; 1024 rows 43 and 35; bf16 8192 x 65536
// 261 and 191).
Cut cut_rows(int32_t dtype, int64_t rows, int64_t V) {
    const int64_t b = type_size(dtype), vecs = V * b / 16;   // at most, whatever the alignment
    if (vecs <= 1024 * 13 || rows == 0) return held_by(vecs, 1, (int32_t)V);
    int64_t pieces = ((V * b + 127) / 128 + kHeldLines - 1) / kHeldLines;
    const int64_t more = rows < kPlaces ? kPlaces / rows : 1, most = vecs / kShortPiece;
    if (pieces < more) pieces = more < most ? more : most;
    return in_pieces(V, b, pieces);
}

template <int DT, bool kTop, bool kPieces>
void score_launch(const ScoreArgs& a, const Cut& c, hipStream_t st) {
    const int64_t n = a.rows * a.pieces;
    const dim3 rows((unsigned)n), quads((unsigned)((n + 3) / 4));
    if (!kPieces && c.threads == 64) score_rows<DT, 64, 8, kTop, false><<<quads, 256, 0, st>>>(a);
    else if (c.threads == 256) score_rows<DT, 256, 8, kTop, kPieces><<<rows, 256, 0, st>>>(a);
    else if (c.held == 8) score_rows<DT, 512, 8, kTop, kPieces><<<rows, 512, 0, st>>>(a);
    else if (c.threads == 512) score_rows<DT, 512, 13, kTop, kPieces><<<rows, 512, 0, st>>>(a);
    else score_rows<DT, 1024, 13, kTop, kPieces><<<rows, 1024, 0, st>>>(a);
}

}  // namespace

}  // namespace gmc

using namespace gmc;

extern "C" {

int64_t gmc_token_scores_workspace(int32_t dtype, int64_t R, int64_t T, int64_t V, int32_t top) {
    if (!known_type(dtype) || R < 0 || T < 0 || V < 1 || V > 0x3fffffff || top < 0 || top > kMostTop || top > V) return -1;
    if (T > 0 && R > kMostRows / T) return -1;
    const int64_t rows = R * T;
    const Cut c = cut_rows(dtype, rows, V);
    if (rows > kMostRows / c.pieces) return -1;   // more than a launch has (and than any memory holds)
    return c.pieces == 1 ? 0 : rows * c.pieces * ((int64_t)sizeof(float4) + 8 * top);
}

gmc_status gmc_token_scores(void* hip_stream, int32_t dtype, int64_t R, int64_t T, int64_t V, const void* logits_dev,
                            int64_t seq_pitch, int64_t tok_pitch, const int64_t* labels_dev, int64_t label_pitch,
                            int64_t ignore, int32_t top, double temperature, float* logp_dev, float* entropy_dev,
                            float* top_logp_dev, int64_t* top_ids_dev, float* norm_dev, void* workspace_dev,
                            int64_t workspace_bytes) {
    const char* me = "gmc_token_scores";
    const gmc_status ok = logits_check(me, dtype, R, T, V, logits_dev, seq_pitch, tok_pitch, nullptr, 0, 0, labels_dev,
                                       label_pitch, true);
    if (ok != GMC_OK) return ok;
    if (top < 0 || top > kMostTop || top > V) return op_error(GMC_EINVAL, me, "top must be in 0 to 32 and no more than V");
    if (!(temperature > 0.0 && isfinite(temperature) && finite_f32(1.4426950408889634 / temperature)))
        return op_error(GMC_EINVAL, me, "temperature must be > 0 and finite, log2(e) / temperature finite in fp32");
    if (R == 0 || T == 0) return GMC_OK;
    if (!entropy_dev || !norm_dev || (labels_dev && !logp_dev) || (top && (!top_logp_dev || !top_ids_dev)))
        return op_error(GMC_EINVAL, me, "NULL argument");
    const int64_t rows = R * T, need = gmc_token_scores_workspace(dtype, R, T, V, top), b = type_size(dtype);
    if (need < 0) return op_error(GMC_EINVAL, me, "more rows and pieces of rows than a launch has");
    if (need && (!workspace_dev || workspace_bytes < need)) return op_error(GMC_EINVAL, me, "the workspace is too small");
    if (need && (reinterpret_cast<uintptr_t>(workspace_dev) & 15u))
        return op_error(GMC_EINVAL, me, "the workspace is not 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(norm_dev) & 7u) return op_error(GMC_EINVAL, me, "norm is not 8-byte aligned");
    if (!apart({{labels_dev ? logp_dev : nullptr, rows * 4}, {entropy_dev, rows * 4}, {norm_dev, rows * 8},
                {top ? top_logp_dev : nullptr, rows * top * 4}, {top ? top_ids_dev : nullptr, rows * top * 8},
                {need ? workspace_dev : nullptr, need}},
               {{logits_dev, rows_span(R, T, V, seq_pitch, tok_pitch, b)}, {labels_dev, rows_span(R, 1, T, label_pitch, 0, 8)}}))
        return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Cut c = cut_rows(dtype, rows, V);
    ScoreArgs a{};
    a.logits = logits_dev;
    a.seq = seq_pitch;
    a.tok = tok_pitch;
    a.labels = labels_dev;
    a.label_pitch = label_pitch;
    a.ignore = ignore;
    a.T = T;
    a.rows = rows;
    a.V = (int32_t)V;
    a.piece = c.piece;
    a.pieces = c.pieces;
    a.top = top;
    a.L = (float)(1.4426950408889634 / temperature);
    a.inv_tau = (float)(1.0 / temperature);
    a.logp = labels_dev ? logp_dev : nullptr;
    a.entropy = entropy_dev;
    a.top_logp = top_logp_dev;
    a.top_ids = top_ids_dev;
    a.norm = norm_dev;
    a.part = static_cast<float4*>(workspace_dev);
    a.keys = reinterpret_cast<uint64_t*>(a.part + rows * c.pieces);
    GMC_BY_TYPE(dtype, {
        if (c.pieces == 1) {
            if (top) score_launch<DT, true, false>(a, c, st);
            else score_launch<DT, false, false>(a, c, st);
        } else {
            if (top) score_launch<DT, true, true>(a, c, st);
            else score_launch<DT, false, true>(a, c, st);
            score_join<DT><<<dim3((unsigned)rows), 256, 0, st>>>(a);
        }
    });
    return op_launched(me);
}

gmc_status gmc_token_scores_backward(void* hip_stream, int32_t dtype, int64_t R, int64_t T, int64_t V,
                                     const void* logits_dev, int64_t seq_pitch, int64_t tok_pitch,
                                     const int64_t* labels_dev, int64_t label_pitch, int64_t ignore, int32_t top,
                                     double temperature, const float* norm_dev, const float* entropy_dev,
                                     const float* dlogp_dev, const float* dentropy_dev, const int64_t* top_ids_dev,
                                     const float* dtop_dev, void* grad_dev, int64_t grad_seq, int64_t grad_tok) {
    const char* me = "gmc_token_scores_backward";
    const gmc_status ok = logits_check(me, dtype, R, T, V, logits_dev, seq_pitch, tok_pitch, grad_dev, grad_seq, grad_tok,
                                       labels_dev, label_pitch, true);
    if (ok != GMC_OK) return ok;
    if (top < 0 || top > kMostTop) return op_error(GMC_EINVAL, me, "top must be in 0 to 32");
    if (!(temperature > 0.0 && isfinite(temperature) && finite_f32(1.4426950408889634 / temperature)))
        return op_error(GMC_EINVAL, me, "temperature must be > 0 and finite, log2(e) / temperature finite in fp32");
    if (dlogp_dev && !labels_dev) return op_error(GMC_EINVAL, me, "dlogp needs labels");
    if (R == 0 || T == 0) return GMC_OK;
    if (!grad_dev || !norm_dev || (dentropy_dev && !entropy_dev) || (top && (!top_ids_dev || !dtop_dev)))
        return op_error(GMC_EINVAL, me, "NULL argument");
    if (reinterpret_cast<uintptr_t>(norm_dev) & 7u) return op_error(GMC_EINVAL, me, "norm is not 8-byte aligned");
    const int64_t rows = R * T, b = type_size(dtype);
    if (!apart({{grad_dev, rows_span(R, T, V, grad_seq, grad_tok, b)}},
               {{labels_dev, rows_span(R, 1, T, label_pitch, 0, 8)}, {norm_dev, rows * 8}, {entropy_dev, rows * 4},
                {dlogp_dev, rows * 4}, {dentropy_dev, rows * 4}, {top ? top_ids_dev : nullptr, rows * top * 8},
                {top ? dtop_dev : nullptr, rows * top * 4}}))
        return op_error(GMC_EINVAL, me, "the gradient overlaps another input than the logits");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    SlopeArgs a{};
    a.logits = logits_dev;
    a.grad = grad_dev;
    a.seq = seq_pitch;
    a.tok = tok_pitch;
    a.grad_seq = grad_seq;
    a.grad_tok = grad_tok;
    a.labels = labels_dev;
    a.label_pitch = label_pitch;
    a.ignore = ignore;
    a.T = T;
    a.rows = rows;
    a.V = (int32_t)V;
    a.piece = (int32_t)V;
    a.pieces = 1;
    a.top = top;
    a.L = (float)(1.4426950408889634 / temperature);
    a.inv_tau = (float)(1.0 / temperature);
    a.norm = norm_dev;
    a.entropy = entropy_dev;
    a.dlogp = dlogp_dev;
    a.dentropy = dentropy_dev;
    a.top_ids = top_ids_dev;
    a.dtop = dtop_dev;
    const int64_t vecs = V * b / 16;
    if (rows < kPlaces && vecs > kShortPiece) {
        const int64_t more = kPlaces / rows, most = vecs / (kShortPiece / 2);
        const Cut c = in_pieces(V, b, more < most ? more : most);
        a.piece = c.piece;
        a.pieces = c.pieces;
    }
    const int64_t groups = rows * a.pieces;
    GMC_BY_TYPE(dtype, {
        if (vecs <= 64 * 8) score_gradient<DT, 64><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, st>>>(a);
        else if (vecs <= 2048 || a.pieces > 1) score_gradient<DT, 512><<<dim3((unsigned)groups), 512, 0, st>>>(a);
        else score_gradient<DT, 1024><<<dim3((unsigned)groups), 1024, 0, st>>>(a);
    });
    return op_launched(me);
}

}  // extern "C"
