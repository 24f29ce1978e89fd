// Device side shared by the block operators: element types, loads and stores
// of eight elements at any address, and sums over a workgroup.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace fsdp_block {

using bf16 = __bf16;
using f16 = _Float16;

// Eight elements, at the alignment of one: gfx950 takes a 16-byte access at any
// address, at nearly the rate of an aligned one.
template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(sizeof(T)))) any {
        type v;
    };
};

// Eight elements as they lie in memory.
template <typename T>
using Eight = typename Vec8<T>::type;

template <typename T>
__device__ __forceinline__ Eight<T> load8(const T* p) {
    return reinterpret_cast<const typename Vec8<T>::any*>(p)->v;
}
// The same of what is read once: past the caches.
template <typename T>
__device__ __forceinline__ Eight<T> load8_once(const T* p) {
    typedef Eight<T> any __attribute__((aligned(sizeof(T))));
    return __builtin_nontemporal_load(reinterpret_cast<const any*>(p));
}
template <typename T>
__device__ __forceinline__ void store8(T* p, Eight<T> v) {
    reinterpret_cast<typename Vec8<T>::any*>(p)->v = v;
}

// The first n of eight elements, zeros after them.
template <typename T>
__device__ __forceinline__ Eight<T> load_some(const T* p, int n) {
    if (n >= 8) return load8(p);
    Eight<T> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : T(0.f);
    return v;
}
// Rounds to nearest even and stores the first n.
template <typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&in)[8]) {
    Eight<T> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = T(in[i]);
    if (n >= 8) return store8(p, v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
}

// Reductions over a wave in six steps through the lanes' own data paths (DPP):
// four within rows of 16 lanes, two that pass a row's last lane on.  The result
// is that of lane 63, for all lanes.  The order of additions is fixed: results do
// not depend on timing.
template <int kCtrl, int kRows>
__device__ __forceinline__ float lanes_moved(float v, float none) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), kCtrl,
                                                                 kRows, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += lanes_moved<0x111, 0xf>(v, 0.f);        // from 1, 2, 4, 8 lanes below
    v += lanes_moved<0x112, 0xf>(v, 0.f);
    v += lanes_moved<0x114, 0xf>(v, 0.f);
    v += lanes_moved<0x118, 0xf>(v, 0.f);
    v += lanes_moved<0x142, 0xa>(v, 0.f);        // rows 0 and 2 into 1 and 3
    v += lanes_moved<0x143, 0xc>(v, 0.f);        // row 1 into 2 and 3
    return last_lane(v);
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, lanes_moved<0x111, 0xf>(v, v));
    v = fmaxf(v, lanes_moved<0x112, 0xf>(v, v));
    v = fmaxf(v, lanes_moved<0x114, 0xf>(v, v));
    v = fmaxf(v, lanes_moved<0x118, 0xf>(v, v));
    v = fmaxf(v, lanes_moved<0x142, 0xa>(v, v));
    v = fmaxf(v, lanes_moved<0x143, 0xc>(v, v));
    return last_lane(v);
}

// Sums of kN values over a workgroup of kThreads, for all threads.  `part`
// holds kN * kThreads / 64 floats; calls that follow each other take different
// ones, or a barrier between them.
template <int kThreads, int kN>
__device__ __forceinline__ void group_sum(float (&v)[kN], float* part) {
    constexpr int kWaves = kThreads / 64;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = wave_sum(v[i]);
    if constexpr (kWaves > 1) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < kN; ++i) part[i * kWaves + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += part[i * kWaves + w];
            v[i] = s;
        }
    }
}

}  // namespace fsdp_block
