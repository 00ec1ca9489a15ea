// What the worker-side operators (gmc_dropout.hip, gmc_norm.hip, gmc_loss.hip)
// share: element types, 16-byte accesses at any element alignment, wavefront
// reductions, and the entry points' error reporting.  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/gmc.h"

namespace gmc {

// Records the message gmc_last_error(NULL) returns and passes the status on;
// never throws (the entry points are C).  Defined in gmc_api.hip.
gmc_status op_error(gmc_status st, const char* where, const char* what) noexcept;

// The launches' error, if any, as a status.
inline gmc_status op_launched(const char* where) noexcept {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GMC_OK : op_error(GMC_EDEVICE, where, hipGetErrorString(e));
}

inline bool known_type(int32_t dtype) { return dtype == GMC_F32 || dtype == GMC_BF16 || dtype == GMC_F16; }
inline int64_t type_size(int32_t dtype) { return dtype == GMC_F32 ? 4 : 2; }

// Whether the byte ranges [a, a + an) and [b, b + bn) share a byte.
inline bool overlap(const void* a, int64_t an, const void* b, int64_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return an > 0 && bn > 0 && x < y + (uintptr_t)bn && y < x + (uintptr_t)an;
}

// A buffer of a call; one that is not there has no bytes.
struct Span {
    const void* p;
    int64_t bytes;
    Span(const void* q, int64_t n) : p(q), bytes(q ? n : 0) {}
};

// Whether each output is apart from the other outputs and from the inputs.
inline bool apart(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
    for (const Span* o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Span* q = o + 1; q != outputs.end(); ++q)
            if (overlap(o->p, o->bytes, q->p, q->bytes)) return false;
        for (const Span& i : inputs)
            if (overlap(o->p, o->bytes, i.p, i.bytes)) return false;
    }
    return true;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// A vector of B bytes, 16 or one element's, that may sit at any element boundary:
// gfx950 takes 16-byte global accesses at any alignment; a wavefront's then touch
// one cache line more.
template <int B>
struct Raw;
template <>
struct Raw<16> {
    typedef uint32_t V __attribute__((ext_vector_type(4)));
};
template <>
struct Raw<4> {
    typedef uint32_t V;
};
template <>
struct Raw<2> {
    typedef uint16_t V;
};

template <int DT>
struct Elem;

// One element type: its storage, conversions of single values and of pairs
// packed in a word.  Rounding to 16 bits is to nearest, ties to even, once,
// from the 32-bit result.
template <>
struct Elem<GMC_F32> {
    typedef float T;
    static constexpr int kSize = 4;
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <>
struct Elem<GMC_BF16> {
    typedef __bf16 T;
    static constexpr int kSize = 2;
    static __device__ __forceinline__ float up(__bf16 v) { return (float)v; }
    static __device__ __forceinline__ __bf16 down(float v) { return (__bf16)v; }
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        f32x2 v;
        v.x = a;
        v.y = b;
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    }
};
template <>
struct Elem<GMC_F16> {
    typedef _Float16 T;
    static constexpr int kSize = 2;
    static __device__ __forceinline__ float up(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 down(float v) { return (_Float16)v; }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w).x; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w).y; }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        f32x2 v;
        v.x = a;
        v.y = b;
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
};

// N consecutive elements as raw bits, loaded and stored in one access.
template <int DT, int N>
struct Vec {
    typedef typename Elem<DT>::T T;
    static constexpr int kBytes = N * Elem<DT>::kSize;
    typedef typename Raw<kBytes>::V V;
    typedef V U __attribute__((aligned(Elem<DT>::kSize)));
    V raw;

    static __device__ __forceinline__ Vec load(const T* p) {
        Vec r;
        r.raw = *reinterpret_cast<const U*>(p);
        return r;
    }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<U*>(p) = raw; }
    // The same for data that is touched once (nontemporal).
    static __device__ __forceinline__ Vec load_once(const T* p) {
        Vec r;
        r.raw = __builtin_nontemporal_load(reinterpret_cast<const U*>(p));
        return r;
    }
    __device__ __forceinline__ void store_once(T* p) const { __builtin_nontemporal_store(raw, reinterpret_cast<U*>(p)); }

    __device__ __forceinline__ uint32_t word(int i) const {
        if constexpr (kBytes <= 4) return (uint32_t)raw;
        else return raw[i];
    }
    __device__ __forceinline__ void set_word(int i, uint32_t w) {
        if constexpr (kBytes <= 4) raw = (V)w;
        else raw[i] = w;
    }
    __device__ __forceinline__ void unpack(float (&f)[N]) const {
        if constexpr (DT == GMC_F32) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __uint_as_float(word(i));
        } else if constexpr (N == 1) {
            f[0] = Elem<DT>::lo(word(0));
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                f[2 * i] = Elem<DT>::lo(word(i));
                f[2 * i + 1] = Elem<DT>::hi(word(i));
            }
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[N]) {
        if constexpr (DT == GMC_F32) {
#pragma unroll
            for (int i = 0; i < N; ++i) set_word(i, __float_as_uint(f[i]));
        } else if constexpr (N == 1) {
            raw = (V)(Elem<DT>::pack(f[0], 0.0f) & 0xffffu);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) set_word(i, Elem<DT>::pack(f[2 * i], f[2 * i + 1]));
        }
    }
};

// Sums and maxima over the 64 lanes of a wavefront, the result in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// The work of workgroup `index` of `total`, so dealt that each XCD has a run of
// neighbours: workgroups go to the 8 XCDs in turn, each with a cache of its own.
__device__ __forceinline__ int64_t xcd_run(unsigned index, unsigned total) {
    const unsigned x = index & 7u, j = index >> 3, q = total >> 3, r = total & 7u;
    return (int64_t)x * q + (x < r ? x : r) + j;
}

constexpr float kLog2e = 1.44269504088896341f;

// 2^x by the hardware instruction (1 ulp; results below 2^-126 are zero).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Calls f with the compile-time element type of dtype.
#define GMC_BY_TYPE(dtype, ...)                                          \
    do {                                                                 \
        if ((dtype) == GMC_F32) {                                        \
            constexpr int DT = GMC_F32;                                  \
            __VA_ARGS__;                                                 \
        } else if ((dtype) == GMC_BF16) {                                \
            constexpr int DT = GMC_BF16;                                 \
            __VA_ARGS__;                                                 \
        } else {                                                         \
            constexpr int DT = GMC_F16;                                  \
            __VA_ARGS__;                                                 \
        }                                                                \
    } while (0)

}  // namespace gmc
