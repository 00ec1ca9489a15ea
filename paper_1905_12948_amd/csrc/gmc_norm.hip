// Group norm with its activation over channels-last images, forward and
// backward (gmc_group_norm and gmc_group_norm_backward in include/gmc.h).
//
//   hat = (x - mean) rstd,  z = hat gamma + beta,  y = act(z)
//   dz = dy act'(z),  dgamma = sum dz hat,  dbeta = sum dz  (images, pixels)
//   dx = rstd (gamma dz - (s1 + hat s2) / m),  s1 = sum gamma dz,
//   s2 = sum gamma dz hat over the m values of an image's group
//
// A thread owns 16 bytes of neighbouring channels and walks over pixels, so
// that a wavefront reads whole lines of the channels-last layout; sums are
// taken per channel and then folded into groups, so groups may have any width.
//
// What bounds it is the bytes, then, images being small, the fixed work of a
// workgroup.  Held form: one workgroup has all pixels of a block of whole groups in
// its registers: x (and dy) are read once and the result is written once, the floor
// of the bytes.  Split form, for images whose groups do not fit, or fit in slivers
// of lines only: per-channel sums of pieces of the image, joined, and a second
// launch that reads the images again.  bf16, relu: 64 x 28 x 28 x 512 forward 18.8 us
// (5.5 TB/s of x and y), backward 38; 64 x 56 x 56 x 256 forward 47 (4.4 TB/s: two
// rounds of workgroups of 1024 threads, one a CU), backward 90 (split: 515 MB in two
// launches, and a join of 5 us).  Far from the bytes: groups of other widths than a power
// of two up to 64, by the general kernels (64 x 14 x 14 x 384 in 32 groups forward 17 us,
// backward 23, for 3.3 and 4.9 us of bytes; 8 x 32 x 32 x 640 29 and 49 for 3.6 and 5.3);
// images in one wide group (64 x 56 x 56 x 256: split, forward 78 us for 35); images of few
// pixels, a workgroup each and block of channels (16384 x 1 x 768 in 12 groups forward 178 us
// for 8.5, backward 303 for 12.8).  Folded kernels of 16-bit groups of one or two channels and
// the general ones at their most vectors put 8 to 46 registers into scratch memory.
//
// In the backward pass z is formed in the order written, one rounding each.  All
// sums are 32-bit, in a fixed order.
#include <math.h>

#include <type_traits>

#include "gmc_norm_plan.h"
#include "gmc_ops.h"

namespace gmc {

namespace {

__device__ __forceinline__ float activate(float z, int act) {
    if (act == GMC_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == GMC_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + exp2_fast(-kLog2e * z));
    return z;
}

// dy act'(z)
__device__ __forceinline__ float back_act(float dy, float z, int act) {
    if (act == GMC_ACT_RELU) return z > 0.0f ? dy : 0.0f;
    if (act == GMC_ACT_SILU) {
        const float gate = __builtin_amdgcn_rcpf(1.0f + exp2_fast(-kLog2e * z));
        return dy * (gate * (1.0f + z * (1.0f - gate)));
    }
    return dy;
}

__device__ __forceinline__ int group_of(const NormArgs& a, int c) {
    return a.cpg_log2 >= 0 ? c >> a.cpg_log2 : c / a.cpg;
}

// Calls f with the activation as a compile-time constant: one branch around a
// loop over the values instead of one at each.
template <class Loop>
__device__ __forceinline__ void by_act(int act, Loop f) {
    if (act == GMC_ACT_RELU) f(std::integral_constant<int, GMC_ACT_RELU>{});
    else if (act == GMC_ACT_SILU) f(std::integral_constant<int, GMC_ACT_SILU>{});
    else f(std::integral_constant<int, GMC_ACT_NONE>{});
}

// A workgroup's place in its block of channels.
struct Place {
    int cv, r, rows, waves;  // channel vector, pixel row, pixel rows, wavefronts
    bool on;
};

__device__ __forceinline__ Place place(const NormArgs& a) {
    Place p;
    p.cv = threadIdx.x & ((1 << a.tp_log2) - 1);
    p.r = threadIdx.x >> a.tp_log2;
    p.rows = blockDim.x >> a.tp_log2;
    p.waves = blockDim.x >> 6;
    p.on = p.cv < a.tc;
    return p;
}

// chan[c] = the sum over the workgroup's threads of v for channel c.  Lanes of
// one channel vector are folded by shuffles, wavefronts (or, where a channel
// block is wider than a wavefront, pixel rows) through LDS, in a fixed order.
template <int VEC>
__device__ __forceinline__ void channel_sums(float (&v)[VEC], const NormArgs& a, const Place& p, float* part,
                                             float* chan) {
    const int width = VEC << a.tp_log2;
    int slots;
    if (a.tp_log2 < 6) {
        for (int o = 1 << a.tp_log2; o < 64; o <<= 1)
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] += __shfl_xor(v[i], o);
        slots = p.waves;
        const int lane = threadIdx.x & 63;
        if (lane < (1 << a.tp_log2))
#pragma unroll
            for (int i = 0; i < VEC; ++i) part[(threadIdx.x >> 6) * width + lane * VEC + i] = v[i];
    } else {
        slots = p.rows;
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[p.r * width + p.cv * VEC + i] = v[i];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.tc * VEC; c += blockDim.x) {
        float s = 0.0f;
        for (int k = 0; k < slots; ++k) s += part[k * width + c];
        chan[c] = s;
    }
    __syncthreads();
}

// Gives `take` the sum of chan over each group's channels, one wavefront a group.
template <class Take>
__device__ __forceinline__ void group_sums(const float* chan, const NormArgs& a, Take take) {
    for (int g = threadIdx.x >> 6; g < a.gw; g += blockDim.x >> 6) {
        float s = 0.0f;
        for (int c = threadIdx.x & 63; c < a.cpg; c += 64) s += chan[g * a.cpg + c];
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) take(g, s);
    }
    __syncthreads();
}

template <int VEC>
__device__ __forceinline__ void load_params(const NormArgs& a, int c0, bool on, float (&ga)[VEC], float (&be)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        ga[i] = on && a.gamma ? a.gamma[c0 + i] : 1.0f;
        be[i] = on && a.beta ? a.beta[c0 + i] : 0.0f;
    }
}

extern __shared__ float norm_lds[];

template <int DT, int VEC, int KP>
__global__ __launch_bounds__(kHeldThreads) void norm_forward_held(NormArgs a) {
    typedef typename Elem<DT>::T T;
    typedef Vec<DT, VEC> V;
    const Place p = place(a);
    float* part = norm_lds;
    float* chan = part + (((a.tp_log2 < 6 ? p.waves : p.rows) * VEC) << a.tp_log2);
    float* grp = chan + (VEC << a.tp_log2);
    const int64_t n = blockIdx.x / (unsigned)a.blocks;
    const int blk = (int)(blockIdx.x - n * a.blocks);
    const int c0 = blk * a.cb + p.cv * VEC;
    const T* px = static_cast<const T*>(a.x) + n * a.x_image + c0;
    T* py = static_cast<T*>(a.out) + n * a.out_image + c0;
    V xv[KP];
#pragma unroll
    for (int k = 0; k < KP; ++k) {
        const int s = p.r + k * p.rows;
        if (p.on && s < a.S) xv[k] = V::load(px + s * a.x_pixel);
    }
    float ga[VEC], be[VEC], mu[VEC], rs[VEC];
    load_params<VEC>(a, c0, p.on, ga, be);
    float sum[VEC], f[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < KP; ++k)
        if (p.on && p.r + k * p.rows < a.S) {
            xv[k].unpack(f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] += f[i];
        }
    channel_sums<VEC>(sum, a, p, part, chan);
    group_sums(chan, a, [&](int g, float s) {
        grp[g] = a.mean[n * a.G + blk * a.gw + g] = s * a.inv_m;
    });
    int gi[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        gi[i] = p.on ? group_of(a, p.cv * VEC + i) : 0;
        mu[i] = grp[gi[i]];
        sum[i] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < KP; ++k)
        if (p.on && p.r + k * p.rows < a.S) {
            xv[k].unpack(f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = f[i] - mu[i];
                sum[i] = __builtin_fmaf(d, d, sum[i]);
            }
        }
    channel_sums<VEC>(sum, a, p, part, chan);
    group_sums(chan, a, [&](int g, float s) {
        grp[g] = a.rstd[n * a.G + blk * a.gw + g] = 1.0f / sqrtf(s * a.inv_m + a.eps);
    });
#pragma unroll
    for (int i = 0; i < VEC; ++i) rs[i] = grp[gi[i]];
#pragma unroll
    for (int k = 0; k < KP; ++k) {
        const int s = p.r + k * p.rows;
        if (p.on && s < a.S) {
            xv[k].unpack(f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = activate((f[i] - mu[i]) * rs[i] * ga[i] + be[i], a.act);
            xv[k].pack(f);
            xv[k].store(py + s * a.out_pixel);
        }
    }
}

// Mean and rstd of the thread's channels, from [N][G].
template <int VEC>
__device__ __forceinline__ void load_stats(const NormArgs& a, int64_t n, int c0, bool on, float (&mu)[VEC],
                                           float (&rs)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int64_t at = n * a.G + (on ? group_of(a, c0 + i) : 0);
        mu[i] = a.mean[at];
        rs[i] = a.rstd[at];
    }
}

template <int DT, int VEC, int KP>
__global__ __launch_bounds__(kHeldThreads) void norm_backward_held(NormArgs a) {
    typedef typename Elem<DT>::T T;
    typedef Vec<DT, VEC> V;
    const Place p = place(a);
    float* part = norm_lds;
    float* chan = part + (((a.tp_log2 < 6 ? p.waves : p.rows) * VEC) << a.tp_log2);
    float* grp1 = chan + (VEC << a.tp_log2);
    float* grp2 = grp1 + a.gw;
    const int64_t n = blockIdx.x / (unsigned)a.blocks;
    const int blk = (int)(blockIdx.x - n * a.blocks);
    const int c0 = blk * a.cb + p.cv * VEC;
    const T* px = static_cast<const T*>(a.x) + n * a.x_image + c0;
    const T* pd = static_cast<const T*>(a.dy) + n * a.dy_image + c0;
    T* po = static_cast<T*>(a.out) + n * a.out_image + c0;
    V xv[KP], dv[KP];
#pragma unroll
    for (int k = 0; k < KP; ++k) {
        const int s = p.r + k * p.rows;
        if (p.on && s < a.S) {
            xv[k] = V::load(px + s * a.x_pixel);
            dv[k] = V::load(pd + s * a.dy_pixel);
        }
    }
    float ga[VEC], be[VEC], mu[VEC], rs[VEC], s1[VEC], s2[VEC];
    load_params<VEC>(a, c0, p.on, ga, be);
    load_stats<VEC>(a, n, c0, p.on, mu, rs);
#pragma unroll
    for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < KP; ++k)
        if (p.on && p.r + k * p.rows < a.S) {
            float f[VEC], d[VEC];
            xv[k].unpack(f);
            dv[k].unpack(d);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float hat = (f[i] - mu[i]) * rs[i];
                const float dz = back_act(d[i], hat * ga[i] + be[i], a.act);
                s1[i] += dz;
                s2[i] = __builtin_fmaf(dz, hat, s2[i]);
            }
        }
    // per image: this workgroup's channels' sums, for dbeta and dgamma
    channel_sums<VEC>(s1, a, p, part, chan);
    for (int c = threadIdx.x; c < a.cb; c += blockDim.x) {
        const float v = chan[c];
        a.part[n * a.C + blk * a.cb + c] = v;
        chan[c] = a.gamma ? v * a.gamma[blk * a.cb + c] : v;
    }
    __syncthreads();
    group_sums(chan, a, [&](int g, float s) { grp1[g] = s * a.inv_m; });
    channel_sums<VEC>(s2, a, p, part, chan);
    for (int c = threadIdx.x; c < a.cb; c += blockDim.x) {
        const float v = chan[c];
        a.part2[n * a.C + blk * a.cb + c] = v;
        chan[c] = a.gamma ? v * a.gamma[blk * a.cb + c] : v;
    }
    __syncthreads();
    group_sums(chan, a, [&](int g, float s) { grp2[g] = s * a.inv_m; });
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int g = p.on ? group_of(a, p.cv * VEC + i) : 0;
        s1[i] = grp1[g];
        s2[i] = grp2[g];
    }
#pragma unroll
    for (int k = 0; k < KP; ++k) {
        const int s = p.r + k * p.rows;
        if (p.on && s < a.S) {
            float f[VEC], d[VEC];
            xv[k].unpack(f);
            dv[k].unpack(d);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float hat = (f[i] - mu[i]) * rs[i];
                const float dz = back_act(d[i], hat * ga[i] + be[i], a.act);
                f[i] = rs[i] * (dz * ga[i] - __builtin_fmaf(hat, s2[i], s1[i]));
            }
            xv[k].pack(f);
            xv[k].store(po + s * a.out_pixel);
        }
    }
}

// -- held form, groups of a power of two of channels ---------------------------
//
// The same statements with fewer instructions, which bound the general kernels
// above: values are folded into their groups before any exchange between lanes,
// statistics are formed once a group, and the unpacked values stay in registers
// where a thread has few vectors (128 x 32 x 32 x 64 bf16 in 32 groups: forward 25 us
// by the general kernel, 11.7 so; backward 54 and 17).

// Stores a vector, nontemporal where a workgroup's blocks of channels are whole
// lines (64 x 14 x 14 x 1024 bf16: 15.1 -> 12.9 us); partial lines have to meet in
// the cache (64 x 56 x 56 x 64 in 32-byte blocks: 20 us, nontemporal 67).
template <int DT, int VEC>
__device__ __forceinline__ void put(const Vec<DT, VEC>& v, typename Elem<DT>::T* p, int once) {
    if (once) {
        asm volatile("");  // or the compiler makes one ordinary store of the two
        v.store_once(p);
        asm volatile("");
    } else {
        v.store(p);
    }
}

// The sums of F values over the lanes that share them: the pixel lanes and,
// where a group is wider than a vector, its neighbours (`within` lanes).
template <int F>
__device__ __forceinline__ void fold_lanes(float (&v)[F], int across, int within) {
    for (int o = 1; o < within; o <<= 1)
#pragma unroll
        for (int i = 0; i < F; ++i) v[i] += __shfl_xor(v[i], o);
    for (int o = across; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < F; ++i) v[i] += __shfl_xor(v[i], o);
}

// F: groups in a thread's vector (1 where a group has at least as many channels).
//
// The moments come from one look at the values, taken while later loads are under
// way: a thread sums differences from its first value of the group and their
// squares, and the threads' moments are joined about the common mean.  That first
// value is one of the thread's n, so its square about their mean is at most n
// times their variance: the subtraction that leaves the squares about the mean
// loses at most a factor n <= 128 of the 32-bit resolution of its own share, and
// next to nothing where no value stands that far out.
template <int DT, int KP, int F>
__global__ __launch_bounds__(kHeldThreads) void norm_forward_fold(NormArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int VEC = 16 / Elem<DT>::kSize;
    constexpr int W = VEC / F;            // channels of the vector in one of its groups
    constexpr bool kKeep = KP <= 8;
    typedef Vec<DT, VEC> V;
    const Place p = place(a);
    // blocks narrower than a line share it in one XCD's cache
    const int64_t id = xcd_run(blockIdx.x, gridDim.x), n = id / (unsigned)a.blocks;
    const int blk = (int)(id - n * a.blocks);
    const int c0 = blk * a.cb + p.cv * VEC;
    const int within = F == 1 ? a.cpg / VEC : 1;
    const int g0 = F == 1 ? (p.cv * VEC) >> a.cpg_log2 : p.cv * F;  // the thread's first group
    float* part = norm_lds;               // [wavefronts][gw]
    float* stat = part + p.waves * a.gw;  // [2][gw]
    const T* px = static_cast<const T*>(a.x) + n * a.x_image + c0;
    T* py = static_cast<T*>(a.out) + n * a.out_image + c0;
    V xv[KP];
    float x[kKeep ? KP : 1][VEC], f[VEC];
#pragma unroll
    for (int k = 0; k < KP; ++k) {
        const int s = p.r + k * p.rows;
        if (p.on && s < a.S) xv[k] = V::load(px + s * a.x_pixel);
    }
    float ga[VEC], be[VEC], sum[F], sq[F], mu[F], first[F];
    load_params<VEC>(a, c0, p.on, ga, be);
    const int lane = threadIdx.x & 63;
    const bool writer = lane < (1 << a.tp_log2) && p.on && (p.cv & (within - 1)) == 0;
    const int64_t at = n * a.G + blk * a.gw;
    const bool any = p.on && p.r < a.S;
    const float have = any ? (float)(((a.S - 1 - p.r) / p.rows + 1) * W) : 0.0f, inv = any ? 1.0f / have : 0.0f;

#pragma unroll
    for (int i = 0; i < F; ++i) sum[i] = sq[i] = first[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < KP; ++k)
        if (p.on && p.r + k * p.rows < a.S) {
            xv[k].unpack(f);
            if (k == 0)
#pragma unroll
                for (int i = 0; i < F; ++i) first[i] = f[i * W];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = f[i] - first[i / W];
                sum[i / W] += d;
                sq[i / W] = __builtin_fmaf(d, d, sq[i / W]);
            }
            if constexpr (kKeep)
#pragma unroll
                for (int i = 0; i < VEC; ++i) x[k][i] = f[i];
        }
    // sq: the squares about the thread's own mean, which `first` then holds
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const float d = sum[i] * inv;
        sq[i] = fmaxf(__builtin_fmaf(-sum[i], d, sq[i]), 0.0f);
        sum[i] = __builtin_fmaf(have, first[i], sum[i]);
        first[i] += d;
    }
    fold_lanes<F>(sum, 1 << a.tp_log2, within);
    if (writer)
#pragma unroll
        for (int i = 0; i < F; ++i) part[(threadIdx.x >> 6) * a.gw + g0 + i] = sum[i];
    __syncthreads();
    for (int g = threadIdx.x; g < a.gw; g += blockDim.x) {
        float t = 0.0f;
        for (int w = 0; w < p.waves; ++w) t += part[w * a.gw + g];
        stat[g] = a.mean[at + g] = t * a.inv_m;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < F; ++i) {
        mu[i] = p.on ? stat[g0 + i] : 0.0f;
        const float d = first[i] - mu[i];
        sq[i] = __builtin_fmaf(have * d, d, sq[i]);
    }
    fold_lanes<F>(sq, 1 << a.tp_log2, within);
    if (writer)
#pragma unroll
        for (int i = 0; i < F; ++i) part[(threadIdx.x >> 6) * a.gw + g0 + i] = sq[i];
    __syncthreads();
    for (int g = threadIdx.x; g < a.gw; g += blockDim.x) {
        float t = 0.0f;
        for (int w = 0; w < p.waves; ++w) t += part[w * a.gw + g];
        stat[a.gw + g] = a.rstd[at + g] = 1.0f / sqrtf(t * a.inv_m + a.eps);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i) ga[i] *= p.on ? stat[a.gw + g0 + i / W] : 0.0f;
    by_act(a.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < KP; ++k) {
            const int s = p.r + k * p.rows;
            if (p.on && s < a.S) {
                if constexpr (!kKeep) xv[k].unpack(f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float d = (kKeep ? x[kKeep ? k : 0][i] : f[i]) - mu[i / W];
                    f[i] = activate(__builtin_fmaf(d, ga[i], be[i]), decltype(act)::value);
                }
                xv[k].pack(f);
                put<DT, VEC>(xv[k], py + s * a.out_pixel, a.once);
            }
        }
    });
}

// The sums of H values over the lanes o, 2 o, ... < 64 apart, by halves: at each
// step a lane sends the half of its values that its partner keeps, so H values
// cost about H exchanges in all.  Value j of the result v[0 .. left) is value
// first + j of the input; `first` and `left` say which the lane holds.
template <int H>
__device__ __forceinline__ void scatter_sums(float* v, int lane, int across, int o, int& first, int& left) {
    if (o < across) return;
    if constexpr (H > 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < H / 2; ++i) {
            const float send = up ? v[i] : v[i + H / 2], keep = up ? v[i + H / 2] : v[i];
            v[i] = keep + __shfl_xor(send, o);
        }
        first += up ? H / 2 : 0;
        left = H / 2;
        scatter_sums<H / 2>(v, lane, across, o >> 1, first, left);
    } else {
        for (; o >= across; o >>= 1) v[0] += __shfl_xor(v[0], o);
    }
}

// The channels' sums of dz (v[0 .. VEC)) and dz hat (v[VEC ..)) over the
// workgroup: into a.part and a.part2 for dbeta and dgamma, and weighted with gamma
// and summed over their groups, s1 / m and s2 / m, into stat[2][gw].
template <int VEC>
__device__ __forceinline__ void join_back_sums(const NormArgs& a, const Place& p, int64_t n, int blk,
                                               float (&v)[2 * VEC], float* part, float* stat) {
    int first = 0, left = 2 * VEC;
    const int lane = threadIdx.x & 63;
    scatter_sums<2 * VEC>(v, lane, 1 << a.tp_log2, 32, first, left);
    // lanes that differ only in steps taken with one value left hold the same sum
    if (p.on)
#pragma unroll
        for (int j = 0; j < 2 * VEC; ++j)
            if (j < left) {
                const int q = first + j;
                part[((threadIdx.x >> 6) * 2 + q / VEC) * a.cb + p.cv * VEC + (q & (VEC - 1))] = v[j];
            }
    __syncthreads();
    // a thread per channel and sum; a group's channels are neighbouring lanes
    for (int e0 = 0; e0 < 2 * a.cb; e0 += blockDim.x) {  // whole wavefronts, for the exchange
        const int e = e0 + threadIdx.x;
        const bool some = e < 2 * a.cb;
        const int which = e >= a.cb, c = e - which * a.cb;
        float t = 0.0f;
        if (some) {
            for (int w = 0; w < p.waves; ++w) t += part[(w * 2 + which) * a.cb + c];
            (which ? a.part2 : a.part)[n * a.C + blk * a.cb + c] = t;
            if (a.gamma) t *= a.gamma[blk * a.cb + c];
        }
        for (int o = 1; o < a.cpg; o <<= 1) t += __shfl_xor(t, o);
        if (some && (c & (a.cpg - 1)) == 0) stat[which * a.gw + (c >> a.cpg_log2)] = t * a.inv_m;
    }
    __syncthreads();
}

template <int DT, int KP, int F>
__global__ __launch_bounds__(kHeldThreads) void norm_backward_fold(NormArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int VEC = 16 / Elem<DT>::kSize;
    constexpr int W = VEC / F;
    constexpr bool kKeep = KP <= 2;
    typedef Vec<DT, VEC> V;
    const Place p = place(a);
    // blocks narrower than a line share it in one XCD's cache
    const int64_t id = xcd_run(blockIdx.x, gridDim.x), n = id / (unsigned)a.blocks;
    const int blk = (int)(id - n * a.blocks);
    const int c0 = blk * a.cb + p.cv * VEC;
    const int g0 = F == 1 ? (p.cv * VEC) >> a.cpg_log2 : p.cv * F;
    float* part = norm_lds;                   // [wavefronts][2][cb]
    float* stat = part + 2 * p.waves * a.cb;  // [2][gw]
    const T* px = static_cast<const T*>(a.x) + n * a.x_image + c0;
    const T* pd = static_cast<const T*>(a.dy) + n * a.dy_image + c0;
    T* po = static_cast<T*>(a.out) + n * a.out_image + c0;
    V xv[KP], dv[KP];
#pragma unroll
    for (int k = 0; k < KP; ++k) {
        const int s = p.r + k * p.rows;
        if (p.on && s < a.S) {
            xv[k] = V::load(px + s * a.x_pixel);
            dv[k] = V::load(pd + s * a.dy_pixel);
        }
    }
    float ga[VEC], be[VEC], mu[F], rs[F], v[2 * VEC], f[VEC], d[VEC];
    float xs[kKeep ? KP : 1][VEC], dzs[kKeep ? KP : 1][VEC];
    load_params<VEC>(a, c0, p.on, ga, be);
    const int64_t at = n * a.G + blk * a.gw;
#pragma unroll
    for (int i = 0; i < F; ++i) {
        mu[i] = p.on ? a.mean[at + g0 + i] : 0.0f;
        rs[i] = p.on ? a.rstd[at + g0 + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) v[i] = 0.0f;
    // dz as raw bits of dy's type: relu's is dy or zero, exactly
    by_act(a.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
#pragma unroll
        for (int k = 0; k < KP; ++k)
            if (p.on && p.r + k * p.rows < a.S) {
                xv[k].unpack(f);
                dv[k].unpack(d);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float c = f[i] - mu[i / W], hat = c * rs[i / W];
                    if constexpr (kAct != GMC_ACT_NONE) d[i] = back_act(d[i], hat * ga[i] + be[i], kAct);
                    v[i] += d[i];
                    v[VEC + i] = __builtin_fmaf(d[i], hat, v[VEC + i]);
                    if constexpr (kKeep) {
                        xs[k][i] = c;
                        dzs[k][i] = d[i];
                    }
                }
                if constexpr (!kKeep && kAct == GMC_ACT_RELU) dv[k].pack(d);
            }
    });
    join_back_sums<VEC>(a, p, n, blk, v, part, stat);
    // dx = rstd (gamma dz - s1/m - hat s2/m) = (rstd gamma) dz + (x - mean) b + c
    float gb[F], gc[F];
#pragma unroll
    for (int i = 0; i < F; ++i) {
        gc[i] = p.on ? -rs[i] * stat[g0 + i] : 0.0f;
        gb[i] = p.on ? -rs[i] * rs[i] * stat[a.gw + g0 + i] : 0.0f;
    }
    by_act(a.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
#pragma unroll
        for (int k = 0; k < KP; ++k) {
            const int s = p.r + k * p.rows;
            if (p.on && s < a.S) {
                if constexpr (!kKeep) {
                    xv[k].unpack(f);
                    dv[k].unpack(d);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int g = i / W;
                    float c, dz;
                    if constexpr (kKeep) {
                        c = xs[k][i];
                        dz = dzs[k][i];
                    } else {
                        c = f[i] - mu[g];
                        dz = d[i];
                        if constexpr (kAct == GMC_ACT_SILU) dz = back_act(dz, c * rs[g] * ga[i] + be[i], kAct);
                    }
                    f[i] = __builtin_fmaf(dz, rs[g] * ga[i], __builtin_fmaf(c, gb[g], gc[g]));
                }
                xv[k].pack(f);
                put<DT, VEC>(xv[k], po + s * a.out_pixel, a.once);
            }
        }
    });
}

// -- split form ---------------------------------------------------------------

// Workgroup (channel block, chunk, image) of the split kernels.  Pixels are counted from
// the chunk's first: an image's own numbers end at 2^31 - 1, where a step past them wraps.
struct Piece {
    int64_t n, first;
    int c0, pixels, chunk;
};

template <int VEC>
__device__ __forceinline__ Piece piece(const NormArgs& a, Place& p, unsigned before = 0) {
    Piece q;
    const unsigned per = (unsigned)(a.chunks * a.cblocks), id = (unsigned)xcd_run(blockIdx.x - before, gridDim.x - before);
    q.n = id / per;
    const unsigned rest = id - (unsigned)q.n * per;
    q.chunk = (int)(rest / (unsigned)a.cblocks);
    const int cblk = (int)(rest - (unsigned)q.chunk * a.cblocks);
    const int tv = cblk * a.tc + p.cv;
    q.c0 = tv * VEC;
    p.on = p.on && q.c0 < a.C;
    q.first = (int64_t)q.chunk * a.chunk;
    q.pixels = a.S - q.first < a.chunk ? (int)(a.S - q.first) : a.chunk;
    return q;
}

// Per (image, chunk, channel): the mean and the sum of squares about it.  A
// thread sums differences from its first pixel's value, one of the n values
// themselves: n times their variance is at least that value's own square about the
// mean, so the subtraction below loses at most a factor n, the few dozen pixels a
// thread has, of the 32-bit resolution, and nothing where levels are far from zero.
template <int DT, int VEC>
__global__ __launch_bounds__(kSplitThreads) void norm_moments(NormArgs a) {
    typedef typename Elem<DT>::T T;
    typedef Vec<DT, VEC> V;
    Place p = place(a);
    const Piece q = piece<VEC>(a, p);
    float* part = norm_lds;
    float* chan = part + (((a.tp_log2 < 6 ? p.waves : p.rows) * VEC) << a.tp_log2);
    const T* px = static_cast<const T*>(a.x) + q.n * a.x_image + q.first * a.x_pixel + q.c0;
    float mean[VEC], sq[VEC], f[VEC], first[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) mean[i] = sq[i] = first[i] = 0.0f;
    float have = 0.0f;
    if (p.on && p.r < q.pixels) {
        V::load(px + p.r * a.x_pixel).unpack(first);
        have = (float)((q.pixels - p.r + p.rows - 1) / p.rows);
    }
    for (int s0 = p.r; s0 < q.pixels && p.on; s0 += kSplitTile * p.rows) {
        V xv[kSplitTile];
#pragma unroll
        for (int k = 0; k < kSplitTile; ++k)
            if (s0 + k * p.rows < q.pixels) xv[k] = V::load(px + (int64_t)(s0 + k * p.rows) * a.x_pixel);
#pragma unroll
        for (int k = 0; k < kSplitTile; ++k)
            if (s0 + k * p.rows < q.pixels) {
                xv[k].unpack(f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float d = f[i] - first[i];
                    mean[i] += d;
                    sq[i] = __builtin_fmaf(d, d, sq[i]);
                }
            }
    }
    const float n1 = have > 0.0f ? 1.0f / have : 0.0f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float d = mean[i] * n1;
        sq[i] = fmaxf(__builtin_fmaf(-mean[i], d, sq[i]), 0.0f);
        mean[i] = first[i] + d;
        f[i] = have * mean[i];
    }
    channel_sums<VEC>(f, a, p, part, chan);
    const float inv = 1.0f / (float)q.pixels;
    const int64_t at = (q.n * a.chunks + q.chunk) * a.C + (q.c0 - p.cv * VEC);
    const int width = a.tc * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float d = mean[i] - chan[p.on ? p.cv * VEC + i : 0] * inv;
        f[i] = sq[i] + have * d * d;
    }
    for (int c = threadIdx.x; c < width; c += blockDim.x)
        if (q.c0 - p.cv * VEC + c < a.C) a.part[at + c] = chan[c] * inv;
    __syncthreads();
    channel_sums<VEC>(f, a, p, part, chan);
    for (int c = threadIdx.x; c < width; c += blockDim.x)
        if (q.c0 - p.cv * VEC + c < a.C) a.part2[at + c] = chan[c];
}

// One wavefront per (image, group): joins the chunks' channel moments.
__global__ __launch_bounds__(kSplitThreads) void norm_join(NormArgs a) {
    const int64_t at = (int64_t)blockIdx.x * (kSplitThreads / 64) + (threadIdx.x >> 6);
    if (at >= a.N * a.G) return;
    const int64_t n = at / a.G;
    const int g = (int)(at - n * a.G), lane = threadIdx.x & 63;
    const unsigned total = (unsigned)(a.chunks * a.cpg);  // below 2^31; e passes it by up to 64
    const float* mean = a.part + n * a.chunks * a.C + (int64_t)g * a.cpg;
    const float* sq = a.part2 + n * a.chunks * a.C + (int64_t)g * a.cpg;
    const float full = (float)a.chunk, rest = (float)(a.S - (a.chunks - 1) * a.chunk);
    float s = 0.0f;
    for (unsigned e = lane; e < total; e += 64) {
        const int k = group_of(a, (int)e), c = (int)e - k * a.cpg;
        s += (k == a.chunks - 1 ? rest : full) * mean[(int64_t)k * a.C + c];
    }
    const float mu = wave_sum(s) * a.inv_m;
    s = 0.0f;
    for (unsigned e = lane; e < total; e += 64) {
        const int k = group_of(a, (int)e), c = (int)e - k * a.cpg;
        const float d = mean[(int64_t)k * a.C + c] - mu;
        s += sq[(int64_t)k * a.C + c] + (k == a.chunks - 1 ? rest : full) * d * d;
    }
    const float var = wave_sum(s) * a.inv_m;
    if (lane == 0) {
        a.mean[at] = mu;
        a.rstd[at] = 1.0f / sqrtf(var + a.eps);
    }
}

template <int DT, int VEC>
__global__ __launch_bounds__(kSplitThreads) void norm_forward_split(NormArgs a) {
    typedef typename Elem<DT>::T T;
    typedef Vec<DT, VEC> V;
    Place p = place(a);
    const Piece q = piece<VEC>(a, p);
    if (!p.on) return;
    const T* px = static_cast<const T*>(a.x) + q.n * a.x_image + q.first * a.x_pixel + q.c0;
    T* py = static_cast<T*>(a.out) + q.n * a.out_image + q.first * a.out_pixel + q.c0;
    float ga[VEC], be[VEC], mu[VEC], rs[VEC], f[VEC];
    load_params<VEC>(a, q.c0, true, ga, be);
    load_stats<VEC>(a, q.n, q.c0, true, mu, rs);
    by_act(a.act, [&](auto act) {
        for (int s0 = p.r; s0 < q.pixels; s0 += 4 * p.rows) {
            V xv[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * p.rows < q.pixels) xv[k] = V::load(px + (int64_t)(s0 + k * p.rows) * a.x_pixel);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * p.rows < q.pixels) {
                    xv[k].unpack(f);
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        f[i] = activate((f[i] - mu[i]) * rs[i] * ga[i] + be[i], decltype(act)::value);
                    xv[k].pack(f);
                    xv[k].store_once(py + (int64_t)(s0 + k * p.rows) * a.out_pixel);
                }
        }
    });
}

// Per (image, chunk, channel): the sums of dz and of dz hat.  Ordinary loads: the next
// launch finds up to 256 MB of what is read here in the cache behind the XCDs'
// (64 x 3136 x 256 bf16: 93 us in all, with nontemporal loads 106).
template <int DT, int VEC>
__global__ __launch_bounds__(kSplitThreads) void norm_back_sums(NormArgs a) {
    typedef typename Elem<DT>::T T;
    typedef Vec<DT, VEC> V;
    Place p = place(a);
    const Piece q = piece<VEC>(a, p);
    float* part = norm_lds;
    float* chan = part + (((a.tp_log2 < 6 ? p.waves : p.rows) * VEC) << a.tp_log2);
    const T* px = static_cast<const T*>(a.x) + q.n * a.x_image + q.first * a.x_pixel + q.c0;
    const T* pd = static_cast<const T*>(a.dy) + q.n * a.dy_image + q.first * a.dy_pixel + q.c0;
    float ga[VEC], be[VEC], mu[VEC], rs[VEC], s1[VEC], s2[VEC];
    load_params<VEC>(a, q.c0, p.on, ga, be);
    load_stats<VEC>(a, q.n, q.c0, p.on, mu, rs);
#pragma unroll
    for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.0f;
    by_act(a.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
        for (int s0 = p.r; s0 < q.pixels && p.on; s0 += 4 * p.rows) {
            V xv[4], dv[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * p.rows < q.pixels) {
                    xv[k] = V::load(px + (int64_t)(s0 + k * p.rows) * a.x_pixel);
                    dv[k] = V::load(pd + (int64_t)(s0 + k * p.rows) * a.dy_pixel);
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * p.rows < q.pixels) {
                    float f[VEC], d[VEC];
                    xv[k].unpack(f);
                    dv[k].unpack(d);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const float hat = (f[i] - mu[i]) * rs[i];
                        if constexpr (kAct != GMC_ACT_NONE) d[i] = back_act(d[i], hat * ga[i] + be[i], kAct);
                        s1[i] += d[i];
                        s2[i] = __builtin_fmaf(d[i], hat, s2[i]);
                    }
                }
        }
    });
    const int64_t at = (q.n * a.chunks + q.chunk) * a.C + (q.c0 - p.cv * VEC);
    const int width = a.tc * VEC;
    channel_sums<VEC>(s1, a, p, part, chan);
    for (int c = threadIdx.x; c < width; c += blockDim.x)
        if (q.c0 - p.cv * VEC + c < a.C) a.part[at + c] = chan[c];
    __syncthreads();
    channel_sums<VEC>(s2, a, p, part, chan);
    for (int c = threadIdx.x; c < width; c += blockDim.x)
        if (q.c0 - p.cv * VEC + c < a.C) a.part2[at + c] = chan[c];
}

// One wavefront per (image, group): s1 / m and s2 / m from the chunks' sums,
// and each channel's sums over the image's chunks, left in the first chunk's row.
__global__ __launch_bounds__(kSplitThreads) void norm_back_join(NormArgs a, float* shared_terms) {
    const int64_t at = (int64_t)blockIdx.x * (kSplitThreads / 64) + (threadIdx.x >> 6);
    if (at >= a.N * a.G) return;
    const int64_t n = at / a.G;
    const int g = (int)(at - n * a.G), lane = threadIdx.x & 63;
    const int64_t base = n * a.chunks * a.C + (int64_t)g * a.cpg;
    // `step` channels side by side, the other lanes on other chunks
    int step = 1;
    while (step < 64 && step < a.cpg) step *= 2;
    float s1 = 0.0f, s2 = 0.0f;
    for (unsigned c0 = 0; c0 < (unsigned)a.cpg; c0 += step) {
        const unsigned c = c0 + (lane & (step - 1));
        float b = 0.0f, w = 0.0f;
        if (c < (unsigned)a.cpg)
            for (int k = lane / step; k < a.chunks; k += 64 / step) {
                b += a.part[base + (int64_t)k * a.C + c];
                w += a.part2[base + (int64_t)k * a.C + c];
            }
        for (int o = step; o < 64; o <<= 1) {
            b += __shfl_xor(b, o);
            w += __shfl_xor(w, o);
        }
        if (lane < step && c < (unsigned)a.cpg) {
            a.part[base + c] = b;
            a.part2[base + c] = w;
            const float ga = a.gamma ? a.gamma[(int64_t)g * a.cpg + c] : 1.0f;
            s1 = __builtin_fmaf(ga, b, s1);
            s2 = __builtin_fmaf(ga, w, s2);
        }
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if (lane == 0) {
        shared_terms[2 * at] = s1 * a.inv_m;
        shared_terms[2 * at + 1] = s2 * a.inv_m;
    }
}

// dgamma and dbeta: the sums over the images of rows of C values, `pitch`
// apart.  16 channels (a 64-byte line of each row) and 16 row slots a workgroup.
__device__ __forceinline__ void sum_params(int block, const float* part, const float* part2, int64_t rows, int64_t pitch,
                                           int32_t C, float* dgamma, float* dbeta) {
    __shared__ float lds[2][kSplitThreads];
    const int c = block * kParamCh + (threadIdx.x & (kParamCh - 1));
    float s1 = 0.0f, s2 = 0.0f;
    if (c < C)
#pragma unroll 4
        for (int64_t r = threadIdx.x / kParamCh; r < rows; r += kSplitThreads / kParamCh) {
            s1 += part[r * pitch + c];
            s2 += part2[r * pitch + c];
        }
    lds[0][threadIdx.x] = s1;
    lds[1][threadIdx.x] = s2;
    __syncthreads();
    for (int h = kSplitThreads / 2; h >= kParamCh; h >>= 1) {
        if (threadIdx.x < h) {
            lds[0][threadIdx.x] += lds[0][threadIdx.x + h];
            lds[1][threadIdx.x] += lds[1][threadIdx.x + h];
        }
        __syncthreads();
    }
    if (threadIdx.x < kParamCh && c < C) {
        if (dbeta) dbeta[c] = lds[0][threadIdx.x];
        if (dgamma) dgamma[c] = lds[1][threadIdx.x];
    }
}

__global__ __launch_bounds__(kSplitThreads) void norm_params(const float* part, const float* part2, int64_t rows,
                                                             int64_t pitch, int32_t C, float* dgamma, float* dbeta) {
    sum_params((int)blockIdx.x, part, part2, rows, pitch, C, dgamma, dbeta);
}

// The first `params` workgroups sum the parameters' gradients, the others are pieces.
template <int DT, int VEC>
__global__ __launch_bounds__(kSplitThreads) void norm_backward_split(NormArgs a, const float* shared_terms, int params,
                                                                     float* dgamma, float* dbeta) {
    typedef typename Elem<DT>::T T;
    typedef Vec<DT, VEC> V;
    if ((int)blockIdx.x < params) {
        sum_params((int)blockIdx.x, a.part, a.part2, a.N, a.chunks * (int64_t)a.C, a.C, dgamma, dbeta);
        return;
    }
    Place p = place(a);
    const Piece q = piece<VEC>(a, p, (unsigned)params);
    if (!p.on) return;
    const T* px = static_cast<const T*>(a.x) + q.n * a.x_image + q.first * a.x_pixel + q.c0;
    const T* pd = static_cast<const T*>(a.dy) + q.n * a.dy_image + q.first * a.dy_pixel + q.c0;
    T* po = static_cast<T*>(a.out) + q.n * a.out_image + q.first * a.out_pixel + q.c0;
    float ga[VEC], be[VEC], mu[VEC], rs[VEC], s1[VEC], s2[VEC];
    load_params<VEC>(a, q.c0, true, ga, be);
    load_stats<VEC>(a, q.n, q.c0, true, mu, rs);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int64_t at = 2 * (q.n * a.G + group_of(a, q.c0 + i));
        s1[i] = shared_terms[at];
        s2[i] = shared_terms[at + 1];
    }
    // as in norm_backward_fold
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        s1[i] = -rs[i] * s1[i];
        s2[i] = -rs[i] * rs[i] * s2[i];
    }
    by_act(a.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
        for (int s0 = p.r; s0 < q.pixels; s0 += 4 * p.rows) {
            V xv[4], dv[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * p.rows < q.pixels) {
                    xv[k] = V::load_once(px + (int64_t)(s0 + k * p.rows) * a.x_pixel);
                    dv[k] = V::load_once(pd + (int64_t)(s0 + k * p.rows) * a.dy_pixel);
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * p.rows < q.pixels) {
                    float f[VEC], d[VEC];
                    xv[k].unpack(f);
                    dv[k].unpack(d);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const float c = f[i] - mu[i];
                        if constexpr (kAct != GMC_ACT_NONE) d[i] = back_act(d[i], c * rs[i] * ga[i] + be[i], kAct);
                        f[i] = __builtin_fmaf(d[i], rs[i] * ga[i], __builtin_fmaf(c, s2[i], s1[i]));
                    }
                    xv[k].pack(f);
                    xv[k].store_once(po + (int64_t)(s0 + k * p.rows) * a.out_pixel);
                }
        }
    });
}

// -- host ---------------------------------------------------------------------

// Images n0, n0 + 1, ... of a, at most n; b: bytes of an element.
NormArgs some_images(NormArgs a, int64_t n0, int64_t n, int64_t b) {
    const int64_t rows = n0 * (a.chunks ? a.chunks : 1) * a.C;
    a.x = static_cast<const char*>(a.x) + n0 * a.x_image * b;
    if (a.dy) a.dy = static_cast<const char*>(a.dy) + n0 * a.dy_image * b;
    a.out = static_cast<char*>(a.out) + n0 * a.out_image * b;
    a.mean += n0 * a.G;
    a.rstd += n0 * a.G;
    if (a.part) {
        a.part += rows;
        a.part2 += rows;
    }
    a.N = a.N - n0 < n ? a.N - n0 : n;
    return a;
}

gmc_status norm_check(const char* me, int32_t dtype, int64_t N, int64_t S, int32_t C, int32_t G, int32_t act) {
    if (!known_type(dtype)) return op_error(GMC_EINVAL, me, "unknown element type");
    if (N < 0 || S < 1 || S > 0x7fffffff || C < 1) return op_error(GMC_EINVAL, me, "need N >= 0, 1 <= S < 2^31, C >= 1");
    if (G < 1 || C % G) return op_error(GMC_EINVAL, me, "C must be a multiple of G >= 1");
    if (act < GMC_ACT_NONE || act > GMC_ACT_SILU) return op_error(GMC_EINVAL, me, "unknown activation");
    if ((int64_t)C * S > (int64_t(1) << 40) || N > (int64_t(1) << 40) / ((int64_t)C * S))
        return op_error(GMC_EINVAL, me, "more than 2^40 elements");
    return GMC_OK;
}

bool image_pitch_ok(int64_t N, int64_t S, int64_t C, int64_t image, int64_t pixel) {
    constexpr int64_t kMost = int64_t(1) << 40;
    if (pixel < C || pixel > kMost / S) return false;
    return N <= 1 || (image >= (S - 1) * pixel + C && image <= kMost / N);
}

int64_t image_span(int64_t N, int64_t S, int64_t C, int64_t image, int64_t pixel, int64_t b) {
    return ((N - 1) * (N > 1 ? image : 0) + (S - 1) * pixel + C) * b;
}

}  // namespace

}  // namespace gmc

using namespace gmc;

#define GMC_NORM_VEC(full, ...)                                       \
    do {                                                              \
        if (pl.vec == (full)) {                                       \
            constexpr int VEC = (full);                               \
            __VA_ARGS__;                                              \
        } else {                                                      \
            constexpr int VEC = 1;                                    \
            __VA_ARGS__;                                              \
        }                                                             \
    } while (0)

#define GMC_NORM_FOLD(...)                                            \
    do {                                                              \
        if (pl.fold == 1) {                                           \
            constexpr int F = 1;                                      \
            __VA_ARGS__;                                              \
        } else if (pl.fold == 2) {                                    \
            constexpr int F = 2;                                      \
            __VA_ARGS__;                                              \
        } else if (pl.fold == 4) {                                    \
            constexpr int F = 4;                                      \
            __VA_ARGS__;                                              \
        } else if constexpr (DT != GMC_F32) {                         \
            constexpr int F = 8;                                      \
            __VA_ARGS__;                                              \
        }                                                             \
    } while (0)

extern "C" {

int64_t gmc_group_norm_workspace(int32_t dtype, int64_t N, int64_t S, int32_t C, int32_t G, int32_t backward) {
    if (norm_check("gmc_group_norm_workspace", dtype, N, S, C, G, GMC_ACT_NONE) != GMC_OK) return -1;
    if (N == 0) return 0;
    NormArgs a{};
    a.N = N;
    a.S = (int32_t)S;
    a.C = C;
    a.G = G;
    const NormPlan pl = norm_plan(a, type_size(dtype), backward != 0);
    if (launch_images(a, pl, backward != 0) < 1) {
        op_error(GMC_EINVAL, "gmc_group_norm_workspace", "more than a launch can have");
        return -1;
    }
    return (int64_t)sizeof(float) * norm_scratch(a, pl, backward != 0);
}

gmc_status gmc_group_norm(void* hip_stream, int32_t dtype, int64_t N, int64_t S, int32_t C, int32_t G,
                          const void* x_dev, int64_t x_image, int64_t x_pixel, const float* gamma_dev,
                          const float* beta_dev, double eps, int32_t act, void* y_dev, int64_t y_image,
                          int64_t y_pixel, float* mean_dev, float* rstd_dev, void* workspace_dev,
                          int64_t workspace_bytes) {
    const char* me = "gmc_group_norm";
    gmc_status ok = norm_check(me, dtype, N, S, C, G, act);
    if (ok != GMC_OK) return ok;
    if (!(eps >= 0.0 && eps <= 1.0)) return op_error(GMC_EINVAL, me, "eps must be in [0, 1]");
    if (N == 0) return GMC_OK;
    if (!x_dev || !y_dev || !mean_dev || !rstd_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    if (!image_pitch_ok(N, S, C, x_image, x_pixel) || !image_pitch_ok(N, S, C, y_image, y_pixel))
        return op_error(GMC_EINVAL, me, "a pitch is shorter than what it steps over");
    const int64_t b = type_size(dtype);
    if (overlap(x_dev, image_span(N, S, C, x_image, x_pixel, b), y_dev, image_span(N, S, C, y_image, y_pixel, b)) &&
        !(x_dev == y_dev && x_pixel == y_pixel && (N == 1 || x_image == y_image)))
        return op_error(GMC_EINVAL, me, "y overlaps x without being it");
    NormArgs a{};
    a.x = x_dev;
    a.out = y_dev;
    a.x_image = x_image;
    a.x_pixel = x_pixel;
    a.out_image = y_image;
    a.out_pixel = y_pixel;
    a.gamma = gamma_dev;
    a.beta = beta_dev;
    a.mean = mean_dev;
    a.rstd = rstd_dev;
    a.N = N;
    a.S = (int32_t)S;
    a.C = C;
    a.G = G;
    a.eps = (float)eps;
    a.act = act;
    const NormPlan pl = norm_plan(a, type_size(dtype), false);
    const int64_t most = launch_images(a, pl, false);
    if (most < 1) return op_error(GMC_EINVAL, me, "more than a launch can have");
    const int64_t need = norm_scratch(a, pl, false);
    if (need && (!workspace_dev || workspace_bytes < need * (int64_t)sizeof(float)))
        return op_error(GMC_EINVAL, me, "the workspace is too small");
    const Span mean(mean_dev, N * G * 4), rstd(rstd_dev, N * G * 4), scratch(workspace_dev, need * 4);
    if (!apart({mean, rstd, scratch, {y_dev, image_span(N, S, C, y_image, y_pixel, b)}},
               {{gamma_dev, C * int64_t(4)}, {beta_dev, C * int64_t(4)}}) ||
        !apart({mean, rstd, scratch}, {{x_dev, image_span(N, S, C, x_image, x_pixel, b)}}))
        return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    a.part = static_cast<float*>(workspace_dev);
    a.part2 = a.part ? a.part + N * a.chunks * (int64_t)C : nullptr;
    for (int64_t n0 = 0; n0 < N; n0 += most) {
        const NormArgs q = some_images(a, n0, most, b);
        const dim3 grid((unsigned)(q.N * (pl.held ? (int64_t)q.blocks : (int64_t)q.chunks * q.cblocks)));
        const dim3 joins((unsigned)((q.N * G + kSplitThreads / 64 - 1) / (kSplitThreads / 64)));
        if (pl.fold) {
            GMC_BY_TYPE(dtype, GMC_NORM_FOLD({
                            if (pl.kp <= 4) norm_forward_fold<DT, 4, F><<<grid, pl.threads, pl.lds, st>>>(q);
                            else if (pl.kp <= 8) norm_forward_fold<DT, 8, F><<<grid, pl.threads, pl.lds, st>>>(q);
                            else norm_forward_fold<DT, kHeldMost, F><<<grid, pl.threads, pl.lds, st>>>(q);
                        }));
        } else if (pl.held) {
            GMC_BY_TYPE(dtype, GMC_NORM_VEC(16 / Elem<DT>::kSize, {
                            if (pl.kp == 4) norm_forward_held<DT, VEC, 4><<<grid, pl.threads, pl.lds, st>>>(q);
                            else norm_forward_held<DT, VEC, kHeldMost><<<grid, pl.threads, pl.lds, st>>>(q);
                        }));
        } else {
            GMC_BY_TYPE(dtype, GMC_NORM_VEC(16 / Elem<DT>::kSize, {
                            norm_moments<DT, VEC><<<grid, pl.threads, pl.lds, st>>>(q);
                            norm_join<<<joins, kSplitThreads, 0, st>>>(q);
                            norm_forward_split<DT, VEC><<<grid, pl.threads, 0, st>>>(q);
                        }));
        }
    }
    return op_launched(me);
}

gmc_status gmc_group_norm_backward(void* hip_stream, int32_t dtype, int64_t N, int64_t S, int32_t C, int32_t G,
                                   const void* dy_dev, int64_t dy_image, int64_t dy_pixel, const void* x_dev,
                                   int64_t x_image, int64_t x_pixel, const float* mean_dev, const float* rstd_dev,
                                   const float* gamma_dev, const float* beta_dev, int32_t act, void* dx_dev,
                                   int64_t dx_image, int64_t dx_pixel, float* dgamma_dev, float* dbeta_dev,
                                   void* workspace_dev, int64_t workspace_bytes) {
    const char* me = "gmc_group_norm_backward";
    gmc_status ok = norm_check(me, dtype, N, S, C, G, act);
    if (ok != GMC_OK) return ok;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (N == 0) {
        if (param_blocks(C) * (int64_t)kSplitThreads > kMostThreads)
            return op_error(GMC_EINVAL, me, "more than a launch can have");
        if (dgamma_dev || dbeta_dev)
            norm_params<<<dim3(param_blocks(C)), kSplitThreads, 0, st>>>(nullptr, nullptr, 0, C, C, dgamma_dev, dbeta_dev);
        return op_launched(me);
    }
    if (!dy_dev || !x_dev || !dx_dev || !mean_dev || !rstd_dev) return op_error(GMC_EINVAL, me, "NULL argument");
    if (!image_pitch_ok(N, S, C, x_image, x_pixel) || !image_pitch_ok(N, S, C, dy_image, dy_pixel) ||
        !image_pitch_ok(N, S, C, dx_image, dx_pixel))
        return op_error(GMC_EINVAL, me, "a pitch is shorter than what it steps over");
    const int64_t b = type_size(dtype);
    const int64_t out_span = image_span(N, S, C, dx_image, dx_pixel, b);
    if ((overlap(x_dev, image_span(N, S, C, x_image, x_pixel, b), dx_dev, out_span) &&
         !(x_dev == dx_dev && x_pixel == dx_pixel && (N == 1 || x_image == dx_image))) ||
        (overlap(dy_dev, image_span(N, S, C, dy_image, dy_pixel, b), dx_dev, out_span) &&
         !(dy_dev == dx_dev && dy_pixel == dx_pixel && (N == 1 || dy_image == dx_image))))
        return op_error(GMC_EINVAL, me, "dx overlaps an input without being it");
    NormArgs a{};
    a.x = x_dev;
    a.dy = dy_dev;
    a.out = dx_dev;
    a.x_image = x_image;
    a.x_pixel = x_pixel;
    a.dy_image = dy_image;
    a.dy_pixel = dy_pixel;
    a.out_image = dx_image;
    a.out_pixel = dx_pixel;
    a.gamma = gamma_dev;
    a.beta = beta_dev;
    a.mean = const_cast<float*>(mean_dev);
    a.rstd = const_cast<float*>(rstd_dev);
    a.N = N;
    a.S = (int32_t)S;
    a.C = C;
    a.G = G;
    a.act = act;
    const NormPlan pl = norm_plan(a, type_size(dtype), true);
    const int64_t most = launch_images(a, pl, true);
    if (most < 1) return op_error(GMC_EINVAL, me, "more than a launch can have");
    const int64_t need = norm_scratch(a, pl, true);
    if (!workspace_dev || workspace_bytes < need * (int64_t)sizeof(float))
        return op_error(GMC_EINVAL, me, "the workspace is too small");
    const Span dgamma(dgamma_dev, C * int64_t(4)), dbeta(dbeta_dev, C * int64_t(4)), scratch(workspace_dev, need * 4);
    if (!apart({dgamma, dbeta, scratch, {dx_dev, out_span}}, {{gamma_dev, C * int64_t(4)}, {beta_dev, C * int64_t(4)},
                                                              {mean_dev, N * G * 4}, {rstd_dev, N * G * 4}}) ||
        !apart({dgamma, dbeta, scratch}, {{x_dev, image_span(N, S, C, x_image, x_pixel, b)},
                                          {dy_dev, image_span(N, S, C, dy_image, dy_pixel, b)}}))
        return op_error(GMC_EINVAL, me, "an output or the workspace overlaps another buffer");
    const int64_t rows = pl.held ? 1 : a.chunks;  // of partial sums, an image
    a.part = static_cast<float*>(workspace_dev);
    a.part2 = a.part + N * rows * C;
    float* shared_terms = a.part2 + N * rows * C;
    // the split form's last launch sums the parameters' gradients too, where it is the only one
    const bool params = dgamma_dev || dbeta_dev, with = params && !pl.held && N <= most;
    for (int64_t n0 = 0; n0 < N; n0 += most) {
        const NormArgs q = some_images(a, n0, most, b);
        const dim3 grid((unsigned)(q.N * (pl.held ? (int64_t)q.blocks : (int64_t)q.chunks * q.cblocks)));
        if (pl.fold) {
            GMC_BY_TYPE(dtype, GMC_NORM_FOLD({
                            if (pl.kp <= 2) norm_backward_fold<DT, 2, F><<<grid, pl.threads, pl.lds, st>>>(q);
                            else if (pl.kp <= 4) norm_backward_fold<DT, 4, F><<<grid, pl.threads, pl.lds, st>>>(q);
                            else norm_backward_fold<DT, kHeldMostBack, F><<<grid, pl.threads, pl.lds, st>>>(q);
                        }));
        } else if (pl.held) {
            GMC_BY_TYPE(dtype, GMC_NORM_VEC(16 / Elem<DT>::kSize, {
                            if (pl.kp == 4) norm_backward_held<DT, VEC, 4><<<grid, pl.threads, pl.lds, st>>>(q);
                            else norm_backward_held<DT, VEC, kHeldMostBack><<<grid, pl.threads, pl.lds, st>>>(q);
                        }));
        } else {
            float* terms = shared_terms + 2 * n0 * G;
            const unsigned first = with ? param_blocks(C) : 0;
            const dim3 joins((unsigned)((q.N * G + kSplitThreads / 64 - 1) / (kSplitThreads / 64)));
            GMC_BY_TYPE(dtype, GMC_NORM_VEC(16 / Elem<DT>::kSize, {
                            norm_back_sums<DT, VEC><<<grid, pl.threads, pl.lds, st>>>(q);
                            norm_back_join<<<joins, kSplitThreads, 0, st>>>(q, terms);
                            norm_backward_split<DT, VEC><<<dim3(grid.x + first), pl.threads, 0, st>>>(
                                q, terms, (int)first, dgamma_dev, dbeta_dev);
                        }));
        }
    }
    if (params && !with)
        norm_params<<<dim3(param_blocks(C)), kSplitThreads, 0, st>>>(a.part, a.part2, N, rows * C, C, dgamma_dev, dbeta_dev);
    return op_launched(me);
}

}  // extern "C"
