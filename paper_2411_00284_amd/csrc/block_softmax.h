// A softmax over rows of logits: the running maximum and sum, and a thread's
// share of a row.
#pragma once

#include "block_device.h"

namespace fsdp_block {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// 2^x by the hardware's instruction, to one unit of the last place; results
// below the smallest normal number are 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The running maximum m and sum s of a softmax, over terms 2^((v - m) c): the
// difference first, so that it is 0 at the maximum whatever its size (v c - m c as
// one multiply-add leaves the rounding of m c, which at a mask of the type's lowest
// value passes any exponent).  A maximum of -inf counts as 0 in the exponents, so
// that threads that hold nothing but -inf (or nothing) keep a sum of 0.
struct Softmax {
    float m = -INFINITY, s = 0.f;
    __device__ static __forceinline__ float base(float m) { return m == -INFINITY ? 0.f : m; }
    // The sum s of maximum m over a maximum whose base is z; a sum of 0 stays one.
    __device__ static __forceinline__ float moved(float s, float m, float z, float c) {
        return s == 0.f ? 0.f : s * exp2_fast((m - z) * c);
    }
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float top = fmaxf(m, m2), z = base(top);
        s = moved(s, m, z, c) + moved(s2, m2, z, c);
        m = top;
    }
};

// log2(v) in 64 bits to about 2^-24: the exponent is exact, the mantissa's
// logarithm is below one half.
__device__ __forceinline__ double log2_of(float v) {
    int e;
    const float f = frexpf(v, &e);                              // v = f 2^e, f in [1/2, 1)
    const bool low = f < 0.70710678f;
    return v == 0.f || !isfinite(v) ? double(__builtin_amdgcn_logf(v))
                                    : double(low ? e - 1 : e) + double(__builtin_amdgcn_logf(low ? f + f : f));
}

// A thread's share of a row: whole 16-byte units, a unit of a thread kThreads
// units from its next, and one of the elements after them.  Units past the row's
// hold -inf, which no maximum and no sum notices.
template <typename T>
struct Unit {
    static constexpr int n = 16 / int(sizeof(T));
    typedef T vec __attribute__((ext_vector_type(n)));
    typedef vec any __attribute__((aligned(sizeof(T))));
    vec v;
    // kLast: the bytes are not needed again.
    template <bool kLast = false>
    __device__ __forceinline__ void load(const T* s, int unit, int units) {
        if (unit < units) {
            const any* const at = reinterpret_cast<const any*>(s + unit * n);
            v = kLast ? __builtin_nontemporal_load(at) : *at;
        } else {
            v = vec(T(-INFINITY));
        }
    }
    // Past the caches: the gradient's next reader comes after the whole of it.
    // (The units that an entry is written into again, through the caches: 528
    // instead of 445 us at 4096 x 128256; all units so: 530.)
    __device__ __forceinline__ static void store(T* s, int unit, vec out) {
        __builtin_nontemporal_store(out, reinterpret_cast<any*>(s + unit * n));
    }
};

constexpr int kTogether = 2;                     // units streamed at a time

template <typename T, int kUnits>
__device__ __forceinline__ void add_units(Softmax& x, const Unit<T> (&u)[kUnits], float c) {
    float most = x.m;
#pragma unroll
    for (int k = 0; k < kUnits; ++k)
#pragma unroll
        for (int i = 0; i < Unit<T>::n; ++i) most = fmaxf(most, float(u[k].v[i]));
    const float z = Softmax::base(most);
    if (most > x.m) x.s = Softmax::moved(x.s, x.m, z, c);
    x.m = most;
#pragma unroll
    for (int k = 0; k < kUnits; ++k)
#pragma unroll
        for (int i = 0; i < Unit<T>::n; ++i) x.s += exp2_fast((float(u[k].v[i]) - z) * c);
}

}  // namespace
}  // namespace fsdp_block
