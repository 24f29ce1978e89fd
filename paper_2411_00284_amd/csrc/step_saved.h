// Matrices in 8 bits (include/fsdp_step.h): what a group's scale is, eight codes
// from eight values and back.
#pragma once

#include "block_device.h"
#include "block_host.h"
#include "fsdp_step.h"

namespace fsdp_block {

// Codes [rows, cols] to values of `dtype`; columns cols .. to_cols - 1 of x become
// zeros.  Arguments have been checked.
fsdp_status restore(const void* codes, int64_t codes_stride, const void* scales, int64_t scales_stride, void* x, int64_t x_stride,
                    int64_t rows, int64_t cols, int64_t to_cols, fsdp_dtype dtype, hipStream_t stream);

namespace {

typedef int8_t i8x8 __attribute__((ext_vector_type(8)));
struct __attribute__((packed, aligned(1))) AnyCodes {
    i8x8 v;
};

constexpr uint32_t kNotFinite = 255;             // a scale's byte

// The scale byte of a group whose largest magnitude has the bits `most`.  With
// M = 1.f 2^E, M / 2^(E - 6) lies in [64, 128) and rounds to 128 from 127.5 on, where
// f's upper seven bits are all ones: half a unit of the seventh carries E up there.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    if (most >= 0x7f800000u) return kNotFinite;
    return max((most + 0x10000u) >> 23, 7u) - 6u;
}
// 2^-e for a byte of 1 .. 249.
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return byte == kNotFinite ? NAN : __builtin_bit_cast(float, byte ? byte << 23 : 0x400000u);
}

// The largest over the four lanes that hold a group: a quad, or (kApart) lanes 16 apart.
template <bool kApart>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    if constexpr (kApart) {
        const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);     // rows of 16 lanes: 0 1 2 3 -> 0 0 2 2, 1 1 3 3
        v = max(a[0], a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);     // halves: 0 1 -> 0 0, 1 1
        return max(b[0], b[1]);
    }
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xf, 0xf, false)));      // lanes 1 0 3 2
    return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xf, 0xf, false)));   // lanes 2 3 0 1
}

__device__ __forceinline__ i8x8 codes_of(const float (&v)[8], uint32_t byte) {
    // A factor of 0 makes an infinity a NaN, whose code is no matter: it is 0.
    const float inverse = scale_inverse(byte == kNotFinite ? 1u : byte);
    i8x8 q;
#pragma unroll
    for (int c = 0; c < 8; ++c) q[c] = byte == kNotFinite ? int8_t(0) : int8_t(int(__builtin_rintf(v[c] * inverse)));
    return q;
}

// A lane's eight columns of a group, whose other columns three more lanes hold (group_max): all
// four are active and call it, those past the row's end with left <= 0.
template <bool kApart = false>
__device__ __forceinline__ void save8(const float (&v)[8], int left, int8_t* codes, uint8_t* scale) {
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (c < left) most = max(most, __builtin_bit_cast(uint32_t, v[c]) & 0x7fffffffu);
    const uint32_t byte = scale_byte(group_max<kApart>(most));
    if (left <= 0) return;
    const i8x8 q = codes_of(v, byte);
    if (left >= 8) {
        reinterpret_cast<AnyCodes*>(codes)->v = q;
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c < left) codes[c] = q[c];
    }
    if ((threadIdx.x & (kApart ? 48 : 3)) == 0) *scale = uint8_t(byte);
}

// Eight values of one group, zeros after the first n.
__device__ __forceinline__ i8x8 load_codes(const int8_t* codes, int n) {
    if (n >= 8) return reinterpret_cast<const AnyCodes*>(codes)->v;
    i8x8 q;
#pragma unroll
    for (int c = 0; c < 8; ++c) q[c] = c < n ? codes[c] : int8_t(0);
    return q;
}
__device__ __forceinline__ i8x8 load_codes_once(const int8_t* codes) {
    typedef i8x8 any __attribute__((aligned(1)));
    return __builtin_nontemporal_load(reinterpret_cast<const any*>(codes));
}

}  // namespace
}  // namespace fsdp_block
