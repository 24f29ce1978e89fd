// The matrix product of operands on the 16-byte grid, its epilogue, and what else
// the product kernels share.
//
// All products of a linear layer (x W^T, dz W, dz^T x) are
// out[i][j] = sum_k A[i][k] B[j][k]; an operand lies row by row (k contiguous:
// "rows") or k by k (i or j contiguous: "columns").
#pragma once

#include "block_device.h"
#include "block_host.h"

namespace fsdp_block {
namespace {

// ------------------------------------------------------------------ elementwise

// Exponentials and reciprocals are the hardware's, each to a unit of the last
// place: an eighth of the instructions of the rounded division and expf, which the
// gradient's elementwise pass would wait for instead of memory (4096 x 14336 with
// SiLU: 133 us instead of 92, with GELU by erfcf 191).  What is below the smallest
// normal number is 0.
//
// kFull (fp32): the exponent is held in two parts, and the activations are off by
// some 12 units of 2^-24 of themselves (GELU's tanh form by the rounding of its
// argument u more, 4 |u|).  Else the exponent's rounding stays in, |x| / 2 units more:
// 7e-6 at GELU of -12, hundreds of times less than the rounding to 16 bits.
template <bool kFull>
__device__ __forceinline__ float exp_of(float x) {
    constexpr float log2e = 1.44269504088896341f, rest = 1.9259629e-8f;      // rest: what log2e misses
    const float hi = log2e * x, e = __builtin_amdgcn_exp2f(hi);
    if constexpr (!kFull) return e;
    const float lo = fmaf(x, rest, fmaf(x, log2e, -hi));
    return fmaf(e, 0.69314718f * lo, e);
}

// 1 / (1 + exp(-z)), and that of -z, neither as a difference (kFull).
template <bool kFull>
__device__ __forceinline__ float sigmoid(float z, float* other) {
    if constexpr (!kFull) {
        const float q = __builtin_amdgcn_rcpf(1.f + exp_of<false>(-z));
        *other = 1.f - q;
        return q;
    }
    const float e = exp_of<true>(fmaxf(-fabsf(z), -150.f)), r = __builtin_amdgcn_rcpf(1.f + e);
    *other = z < 0.f ? r : e * r;
    return z < 0.f ? e * r : r;
}

// The normal distribution at z, and exp(-z^2 / 2).  erfc(x) = exp(-x^2) t P(t) with
// t = 1 / (1 + 0.3 x) for x >= 0; P, of degree 8, is a minimax fit of the relative
// error over x in [0, 10] (5e-7 as computed in fp32); past that erfc is 0 in fp32.
template <bool kFull>
__device__ __forceinline__ float normal_cdf(float z, float* bell) {
    constexpr float c[9] = {0.16918162f, 0.17081371f, 0.14769703f, 0.2172434f, -0.099725366f, 0.55464029f, -0.51802737f, 0.48822719f, -0.13005051f};
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3f * 0.70710678118654752f * fabsf(z));
    float p = c[8];
#pragma unroll
    for (int i = 7; i >= 0; --i) p = p * t + c[i];
    if constexpr (kFull) {
        const float y = fminf(fabsf(z), 20.f), square = y * y, e = exp_of<true>(-0.5f * square);
        *bell = fmaf(e, -0.5f * fmaf(y, y, -square), e);
    } else {
        *bell = exp_of<false>(-0.5f * z * z);
    }
    const float tail = 0.5f * t * p * *bell;
    return z < 0.f ? tail : 1.f - tail;
}

// act(z); 1 + tanh(u) is 2 sigmoid(2u).
template <bool kFull>
__device__ __forceinline__ float act_value(float z, int act) {
    float other;
    switch (act) {
        case FSDP_ACT_RELU: return z != z ? z : fmaxf(z, 0.f);
        case FSDP_ACT_SILU: return z * sigmoid<kFull>(z, &other);
        case FSDP_ACT_GELU: return z * normal_cdf<kFull>(z, &other);
        case FSDP_ACT_GELU_TANH: return z * sigmoid<kFull>(1.5957691216057308f * (z + 0.044715f * z * z * z), &other);
        default: return z;
    }
}

// act(z) and its slope.
template <bool kFull>
__device__ __forceinline__ void act_both(float z, int act, float& value, float& slope) {
    float other;
    switch (act) {
        case FSDP_ACT_RELU:
            value = z != z ? z : fmaxf(z, 0.f);
            slope = z != z ? z : z > 0.f ? 1.f : 0.f;
            return;
        case FSDP_ACT_SILU: {
            const float q = sigmoid<kFull>(z, &other);
            value = z * q;
            slope = q * (1.f + z * other);
            return;
        }
        case FSDP_ACT_GELU: {
            const float cdf = normal_cdf<kFull>(z, &other);
            value = z * cdf;
            slope = cdf + z * (0.39894228040143268f * other);
            return;
        }
        case FSDP_ACT_GELU_TANH: {
            const float q = sigmoid<kFull>(1.5957691216057308f * (z + 0.044715f * z * z * z), &other);
            value = z * q;
            // Past 30 the product of the two is 0, and z^2 may be infinite.
            const float near = fminf(fabsf(z), 30.f);
            slope = q + z * (q * other) * (1.5957691216057308f * (1.f + 0.134145f * near * near));
            return;
        }
        default:
            value = z;
            slope = 1.f;
    }
}

// ------------------------------------------------------------------ arguments

struct Epilogue {
    const void *bias, *times, *residual;
    void *pre, *out;
    int64_t times_stride, residual_stride, pre_stride, out_stride;
    int act;
};

struct Product {
    const void *a, *b;
    int64_t a_stride, b_stride;
    int64_t m, n, k;                 // out [m, n]
    Epilogue e;
    // A product may be cut along k: part s sums k from s * part_k on, and with
    // more than one part each leaves its sums in parts[s] [m, round_up(n, 8)],
    // for join_parts_kernel.
    float* parts;
    int64_t part_k;
    int count;
    int64_t first_i, first_j;        // the tiles begin there and go to m and n
};

// What the epilogue reads for eight columns of a row.
template <typename T>
struct Extras {
    Eight<T> times, residual;
    __device__ __forceinline__ void load(const Epilogue& e, int64_t i, int64_t j, int left) {
        if (e.times) times = load_some(static_cast<const T*>(e.times) + i * e.times_stride + j, left);
        if (e.residual) residual = load_some(static_cast<const T*>(e.residual) + i * e.residual_stride + j, left);
    }
};

template <typename T>
__device__ __forceinline__ Eight<T> load_bias(const Epilogue& e, int64_t j, int left) {
    return e.bias && left > 0 ? load_some(static_cast<const T*>(e.bias) + j, left) : Eight<T>(T(0.f));
}

// z -> out at row i, columns j .. j + 7, of which `left` exist; `z` is the
// product, without the bias.
template <typename T>
__device__ __forceinline__ void finish8(const Epilogue& e, int64_t i, int64_t j, int left, const Eight<T>& bias,
                                        const Extras<T>& x, float (&z)[8]) {
    if (e.bias)
#pragma unroll
        for (int c = 0; c < 8; ++c) z[c] += float(bias[c]);
    if (e.pre) store_some(static_cast<T*>(e.pre) + i * e.pre_stride + j, left, z);
    if (e.act != FSDP_ACT_NONE)
#pragma unroll
        for (int c = 0; c < 8; ++c) z[c] = act_value<sizeof(T) == 4>(z[c], e.act);
    if (e.times)
#pragma unroll
        for (int c = 0; c < 8; ++c) z[c] *= float(x.times[c]);
    if (e.residual)
#pragma unroll
        for (int c = 0; c < 8; ++c) z[c] += float(x.residual[c]);
    store_some(static_cast<T*>(e.out) + i * e.out_stride + j, left, z);
}
template <typename T>
__device__ __forceinline__ void finish8(const Epilogue& e, int64_t i, int64_t j, int left, float (&z)[8]) {
    Extras<T> x;
    x.load(e, i, j, left);
    finish8<T>(e, i, j, left, load_bias<T>(e, j, left), x, z);
}

// The parts' sums, in order, and the epilogue: a thread takes eight columns.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const Product p) {
    const int64_t units = (p.n + 7) / 8, stride = units * 8;
    for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < p.m * units; u += int64_t(gridDim.x) * 256) {
        const int64_t i = u / units, j = u % units * 8;
        float z[8] = {};
        for (int s = 0; s < p.count; ++s) {
            const Eight<float> v = load8(p.parts + (s * p.m + i) * stride + j);
#pragma unroll
            for (int c = 0; c < 8; ++c) z[c] += v[c];
        }
        finish8<T>(p.e, i, j, int(min(p.n - j, int64_t(8))), z);
    }
}

// ------------------------------------------------------------------ matrix cores

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// 16 bytes of A rows and of B rows per lane -> a 32 x 32 tile.  Lane l holds
// row l % 32 of both and the (l / 32)-th 16 bytes of a 32-byte run of k; element
// r of lane l of the tile is at A row 8 (r / 4) + 4 (l / 32) + r % 4, B row l % 32.
__device__ __forceinline__ f32x16 mma(Eight<bf16> a, Eight<bf16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(Eight<f16> a, Eight<f16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// fp32, two k an instruction: a lane's four values are four of them, the same
// for both operands.  A sixteenth of the 16-bit rate.
__device__ __forceinline__ f32x16 mma(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// Tile `id` of a launch: workgroups go to the 8 XCDs in turn, and each XCD has
// an L2 of its own, so an XCD takes a run of tiles; in a run eight tiles of one
// column of tiles follow each other, so that the 32 tiles in flight on an XCD
// share eight strips of A and four of B.
struct TilePlace {
    int row, column, part;
};
__device__ __forceinline__ TilePlace tile_place(unsigned id, unsigned tiles_m, unsigned tiles_n, unsigned count) {
    const unsigned all = tiles_m * tiles_n * count, xcd = id % 8, each = all / 8, more = all % 8;
    id = xcd * each + min(xcd, more) + id / 8;
    const unsigned part = id / (tiles_m * tiles_n);
    id -= part * tiles_m * tiles_n;
    constexpr unsigned kStrip = 8;
    const unsigned strip = id / (kStrip * tiles_n), first = strip * kStrip, rows = min(kStrip, tiles_m - first);
    id -= first * tiles_n;
    return {int(first + id % rows), int(id / rows), int(part)};
}

// ------------------------------------------------------------------ the aligned product

// A kTileM x kTileN tile of out in four waves, each a quarter of it.
//
// k goes by in steps of 128 bytes of a row, a cache line: 64 k of 16 bits, 32 of
// fp32 (with steps of half a line the L2 answers twice the requests: 1170 instead
// of 1300 TFLOP/s at 8192 x 8192 x 8192).  kSteps steps of both operands lie in LDS.  A step is
// worked on in two halves, two matrix instructions deep each, whose operands lie
// in registers: while the matrix cores take one half the registers of the next
// are read.  Once the second half of a step is in registers its place in LDS is
// free for the step kSteps later, which then has the time of kSteps - 1 steps to
// arrive.
// Loads go from memory to LDS without passing registers; out of range they give
// zeros, which is how odd sizes end.  A workgroup barrier a step.
//
// Large products are bound by the matrix cores: 1250 TFLOP/s with both operands by
// rows, 1300 by columns (8192 x 4096 x 14336, bf16, tiles of 256 x 256), where the
// same instructions without loads run at 1460 to 1490 and alone at 1510 to 1530.
// Small ones are bound by the time of a load: more and smaller steps in flight
// (kSteps 4 and 8) in smaller tiles keep more CUs and more of memory busy.
//
// LDS layout, for conflict-free reads: "rows" 128 bytes per row, with the
// 16-byte units of row r exchanged by r / 2; "columns" one run of columns per k,
// its units exchanged by k, read with the transposing load or (fp32) by element.
template <typename T, int kRows, bool kColumns>
struct Operand {
    static constexpr int kSize = int(sizeof(T)), kDeep = 128 / kSize, kUnit = 16 / kSize;   // k of a step, elements of a unit
    static constexpr int kBytes = kRows * 128;         // of a step
    static constexpr int kLoads = kRows / 32;          // per thread and step, 16 bytes each
    static constexpr int kUnits = kRows / kUnit;       // units of one k of "columns"
    // What the units of k are exchanged by.
    __device__ static __forceinline__ int exchange(int k) {
        return kSize == 4 ? (k >> 2 & 1) * 8 : kRows >= 128 ? (k & 3) * 4 : (k & 2) * 2;
    }

    static constexpr int64_t kNowhere = 0xfffffff0u;   // out of any range

    const char* at;            // the step's first byte
    int64_t step;              // bytes from a step to the next
    int64_t left;              // bytes from `at` to the operand's end, in whole units
    uint32_t offset[kLoads];
    int k;                     // this lane's first k of a step ("rows")

    __device__ __forceinline__ Operand(const void* p, int64_t stride, int64_t first, int64_t rows, int64_t k0, int64_t k1) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if constexpr (kColumns) {
            at = static_cast<const char*>(p) + (k0 * stride + first) * kSize;
            step = kDeep * stride * kSize;
            left = (k1 - 1 - k0) * stride * kSize + (rows - first + kUnit - 1) / kUnit * 16;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int unit = (j * 4 + wave) * 64 + lane, kk = unit / kUnits, u = unit % kUnits;
                offset[j] = uint32_t(min(kk * stride * kSize + (u ^ exchange(kk)) * 16, kNowhere));
            }
            k = 0;
        } else {
            at = static_cast<const char*>(p) + (first * stride + k0) * kSize;
            step = 128;
            left = (rows - 1 - first) * stride * kSize + (k1 - k0 + kUnit - 1) / kUnit * 16;
            const int u = lane % 8 ^ (wave % 2 * 4 + lane / 16);
            k = u * kUnit;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int row = (j * 4 + wave) * 8 + lane / 8;
                offset[j] = uint32_t(min(row * stride * kSize + u * 16, kNowhere));
            }
        }
    }

    // Asks for the next step, with `rest` k left, into `lds`.  Offsets are 32 bits from
    // the tile's first byte, and none of the operand's own passes kMost: the host takes no
    // form of larger ones.
    __device__ __forceinline__ void load(char* lds, int64_t rest) {
        typedef __attribute__((address_space(3))) void lds_void;
        constexpr uint32_t kMost = 0x7ffffff0u;
        const uint32_t bytes = rest <= 0 ? 0u : uint32_t(min(left, int64_t(kMost)));
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, int(bytes), 0x00020000);
        const bool mine = kColumns || k < rest;
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)(lds + (j * 4 + (threadIdx.x >> 6)) * 1024), 16,
                                                     int(mine ? offset[j] : uint32_t(kNowhere)), 0, 0, 0);
        at += step;
        left -= step;
    }
};

// The 16 bytes of an operand that a lane gives to a matrix instruction.
template <typename T>
struct LaneUnit {
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
};

// A wave's registers of half a step: kTiles times 32 rows of an operand, in two
// pairs of units.
// (kApart: how many rows lie between the first half of the tiles and the second, over
// what they cover: 0 where they follow each other.)
template <typename T, int kRows, bool kColumns, int kTiles, int kApart = 0>
struct Fragments {
    static constexpr int row_of(int x) { return x * 32 + (x >= kTiles / 2 ? kApart : 0); }
    static constexpr bool kWide = sizeof(T) == 4;
    static constexpr int kPlaces = kColumns ? kTiles : 4;
    static constexpr int kReads = 2 * kTiles * (!kColumns ? 1 : kWide ? 4 : 2);     // LDS instructions
    typename LaneUnit<T>::type v[2][kTiles];
    // This lane's places in a step's LDS, of the wave whose first row is `first`.
    __device__ static __forceinline__ void lane_places(int first, int (&place)[kPlaces]) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int x = 0; x < kPlaces; ++x) {
            if constexpr (!kColumns) {
                place[x] = (first + lane % 32) * 128 + ((2 * x + lane / 32) ^ lane / 2 % 8) * 16;
            } else {
                // 16 bits: the 4 x 16 block of k and columns that 16 lanes point to; fp32: a column of four k.
                const int k = kWide ? lane / 32 * 4 : lane / 32 * 8 + lane % 16 / 4;
                const int byte = kWide ? (first + 32 * x + lane % 32) * 4 : (first + 32 * x + lane / 16 % 2 * 16 + lane % 4 * 4) * 2;
                place[x] = k * kRows * int(sizeof(T)) + (byte ^ Operand<T, kRows, true>::exchange(k) * 16);
            }
        }
    }
    __device__ __forceinline__ void read(const char* lds, const int (&place)[kPlaces], int half) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < kTiles; ++x) {
                if constexpr (!kColumns) {
                    v[h][x] = *reinterpret_cast<const typename LaneUnit<T>::type*>(lds + place[2 * half + h] + row_of(x) * 128);
                } else if constexpr (kWide) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[h][x][i] = *reinterpret_cast<const float*>(lds + place[x] + ((2 * half + h) * 8 + i) * kRows * 4);
                } else {
                    // The transposing load gives lane i of 16 the i-th column of their block.
                    const char* const at = lds + place[x] + (2 * half + h) * 16 * kRows * 2;
                    v[h][x] = __builtin_bit_cast(Eight<T>, __builtin_shufflevector(
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at),
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * kRows * 2)), 0, 1, 2, 3, 4, 5, 6, 7));
                }
            }
    }
};

// What a kind of product has of its own: where B lies, how far apart the columns of a
// wave's tiles are, and what becomes of eight columns of a row.  This is the kind of one
// matrix B and one of out.
struct OneMatrix {
    static constexpr bool kPair = false;         // tiles of kTileN / 2 columns of two matrices
    static constexpr int kRun = 0;               // steps of fp32 after which their sum joins the others', 0: none
    template <typename T, int kTileN, bool kColumnsB>
    using B = Operand<T, kTileN, kColumnsB>;
    template <typename T, int kTileN, bool kColumnsB>
    __device__ static __forceinline__ auto operand(const Product& p, int64_t j0, int64_t k0, int64_t k1) {
        return B<T, kTileN, kColumnsB>(p.b, p.b_stride, j0, p.n, k0, k1);
    }
    template <typename T>
    __device__ static __forceinline__ void store(const Product& p, int64_t i, int64_t j, int left, const float (&z)[8]) {
        store_some(static_cast<T*>(p.e.out) + i * p.e.out_stride + j, left, z);
    }
};

template <typename T, bool kColumnsA, bool kColumnsB, int kTileM, int kTileN, int kSteps, typename Kind, typename Args>
__device__ __forceinline__ void product_tile(const Args& p) {
    using A = Operand<T, kTileM, kColumnsA>;
    using B = typename Kind::template B<T, kTileN, kColumnsB>;
    constexpr int kDeep = A::kDeep;
    constexpr int kA = kTileM / 64, kB = kTileN / 64;            // 32-row tiles of a wave
    // One array per step: their reads and loads are known not to touch each other.
    constexpr int kA4 = kSteps > 2 ? A::kBytes : 16, kB4 = kSteps > 2 ? B::kBytes : 16;
    constexpr int kA8 = kSteps > 4 ? A::kBytes : 16, kB8 = kSteps > 4 ? B::kBytes : 16;
    __shared__ __attribute__((aligned(1024))) char a0[A::kBytes], a1[A::kBytes], a2[kA4], a3[kA4], a4[kA8], a5[kA8], a6[kA8], a7[kA8];
    __shared__ __attribute__((aligned(1024))) char b0[B::kBytes], b1[B::kBytes], b2[kB4], b3[kB4], b4[kB8], b5[kB8], b6[kB8], b7[kB8];
    static_assert(kSteps == 2 || kSteps == 4 || kSteps == 8);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wi = wave / 2 * (kTileM / 2), wj = wave % 2 * (kTileN / 2);
    const TilePlace t = tile_place(blockIdx.x, unsigned((p.m - p.first_i + kTileM - 1) / kTileM), unsigned((p.n - p.first_j + kTileN - 1) / kTileN),
                                   unsigned(p.count));
    const int64_t i0 = p.first_i + int64_t(t.row) * kTileM, j0 = p.first_j + int64_t(t.column) * kTileN;
    const int64_t k0 = t.part * p.part_k, k1 = min(k0 + p.part_k, p.k);
    A a(p.a, p.a_stride, i0, p.m, k0, k1);
    B b = Kind::template operand<T, kTileN, kColumnsB>(p, j0, k0, k1);
    using FA = Fragments<T, kTileM, kColumnsA, kA>;
    using FB = Fragments<T, kTileN, kColumnsB, kB, Kind::kPair ? kTileN / 4 : 0>;
    FA fa[2];
    FB fb[2];
    int pa[FA::kPlaces], pb[FB::kPlaces];
    FA::lane_places(wi, pa);
    FB::lane_places(Kind::kPair ? wj / 2 : wj, pb);
    f32x16 acc[kA][kB] = {};
    // fp32: a sum of few terms, and the sum of those; a term's rounding is then of a small sum.
    constexpr bool kRuns = Kind::kRun > 0 && sizeof(T) == 4;
    static_assert(Kind::kRun % kSteps == 0);
    f32x16 sum[kRuns ? kA : 1][kRuns ? kB : 1] = {};
    int run = 0;
    const auto join = [&] {
#pragma unroll
        for (int x = 0; x < kA; ++x)
#pragma unroll
            for (int y = 0; y < kB; ++y) {
                sum[x][y] += acc[x][y];
                acc[x][y] = f32x16{};
            }
    };

    // Waits for this wave's loads, but for those of the last kLater steps, and
    // its LDS reads; then for the other waves.
    const auto sync = [](auto later) {
        constexpr int n = decltype(later)::value * (A::kLoads + B::kLoads);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 7 << 4);        // vmcnt(n) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    int64_t rest = k1 - k0;                                       // k not yet asked for
    const auto ask = [&](char* la, char* lb) {
        a.load(la, rest);
        b.load(lb, rest);
        rest -= kDeep;
    };
    constexpr int kMma = 2 * kA * kB * (sizeof(T) == 4 ? 4 : 1), kReads = FA::kReads + FB::kReads,
                  kLoads = A::kLoads + B::kLoads;
    // Half a step: the order of issue is LDS reads first, under the matrix
    // instructions, which then have the rest of the half to arrive; the memory
    // loads after them.
    const auto half = [&](const FA& xa, const FB& xb, auto loads) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < kA; ++x)
#pragma unroll
                for (int y = 0; y < kB; ++y) acc[x][y] = mma(xa.v[h][x], xb.v[h][y], acc[x][y]);
        if constexpr (decltype(loads)::value) {
            constexpr int kTurns = kLoads, kEach = kMma / kTurns > 0 ? kMma / kTurns : 1;
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (kReads + kTurns - 1) / kTurns, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
            }
        } else {
            constexpr int kFew = (kReads + kMma / 2 - 1) / (kMma / 2);
#pragma unroll
            for (int i = 0; i < kReads; i += kFew) {
                __builtin_amdgcn_sched_group_barrier(0x100, kFew, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
        }
    };
    // A step that lies in (la, lb), the next one in (ma, mb).
    const auto step = [&](char* la, char* lb, char* ma, char* mb) {
        fa[1].read(la, pa, 1);
        fb[1].read(lb, pb, 1);
        half(fa[0], fb[0], std::false_type());
        sync(std::integral_constant<int, kSteps - 2>());
        ask(la, lb);
        fa[0].read(ma, pa, 0);
        fb[0].read(mb, pb, 0);
        half(fa[1], fb[1], std::true_type());
        __builtin_amdgcn_sched_barrier(0);
    };
    ask(a0, b0);
    ask(a1, b1);
    if constexpr (kSteps > 2) {
        ask(a2, b2);
        ask(a3, b3);
    }
    if constexpr (kSteps > 4) {
        ask(a4, b4);
        ask(a5, b5);
        ask(a6, b6);
        ask(a7, b7);
    }
    sync(std::integral_constant<int, kSteps - 1>());
    fa[0].read(a0, pa, 0);
    fb[0].read(b0, pb, 0);
    // Steps past the end add zeros: the loop takes kSteps at a time.
    for (int64_t left = k1 - k0; left > 0; left -= kDeep * kSteps) {
        if constexpr (kRuns) {
            if (run == Kind::kRun) {
                join();
                run = 0;
            }
            run += kSteps;
        }
        step(a0, b0, a1, b1);
        if constexpr (kSteps == 2) {
            step(a1, b1, a0, b0);
        } else {
            step(a1, b1, a2, b2);
            step(a2, b2, a3, b3);
            if constexpr (kSteps == 4) {
                step(a3, b3, a0, b0);
            } else {
                step(a3, b3, a4, b4);
                step(a4, b4, a5, b5);
                step(a5, b5, a6, b6);
                step(a6, b6, a7, b7);
                step(a7, b7, a0, b0);
            }
        }
    }
    sync(std::integral_constant<int, 0>());                       // nothing more is written to LDS
    if constexpr (kRuns)
#pragma unroll
        for (int x = 0; x < kA; ++x)
#pragma unroll
            for (int y = 0; y < kB; ++y) acc[x][y] += sum[x][y];

    // A wave passes its sums through its own piece of LDS, kTurn tiles at a time,
    // so that a lane gets eight neighbouring columns; every other four rows have
    // their halves of 32 columns exchanged, against conflicts.  What the epilogue
    // reads of kAhead rows is asked for before the first of them is finished.
    // No other wave touches the piece, so no barrier of the workgroup is needed; the fences
    // keep the lanes' writes before the reads of other lanes', and those before the next
    // writes.
    constexpr int kWide = kTileN / 2, kLanes = kWide / 8, kTurn = kA > 1 ? 2 : 1, kStepRows = 64 / kLanes,
                  kAhead = kTurn * 32 / kStepRows < 4 ? kTurn * 32 / kStepRows : 4;
    static_assert(kTurn * 32 * kWide * 4 <= B::kBytes && kA % kTurn == 0 && kTurn * 32 % (kAhead * kStepRows) == 0 &&
                  (kSteps > 2 || A::kBytes == B::kBytes));
    char* const piece = kSteps > 2 ? (wave == 0 ? b0 : wave == 1 ? b1 : wave == 2 ? b2 : b3)
                                    : (wave == 0 ? a0 : wave == 1 ? a1 : wave == 2 ? b0 : b1);
    float* const turn = reinterpret_cast<float*>(piece);
    const auto place = [](int row, int column) { return row * kWide + (column ^ (kWide > 32 ? row / 4 % 2 * 32 : 0)); };
    if constexpr (Kind::kPair) {
        Kind::template finish<T, kWide>(p, t.part, turn, place, i0 + wi, (j0 + wj) / 2, [&](auto each) {
#pragma unroll
            for (int x0 = 0; x0 < kA; x0 += kTurn) {
#pragma unroll
                for (int x = 0; x < kTurn; ++x)
#pragma unroll
                    for (int y = 0; y < kB; ++y)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            turn[place(32 * x + 8 * (r / 4) + 4 * (lane / 32) + r % 4, 32 * y + lane % 32)] = acc[x0 + x][y][r];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                each(32 * x0, 32 * kTurn);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        });
        return;
    }
    const int column = lane % kLanes * 8;
    const int64_t j = j0 + wj + column;
    const int left = int(min(p.n - j, int64_t(8)));
    const Eight<T> bias = kColumnsB ? Eight<T>(T(0.f)) : load_bias<T>(p.e, j, left);
#pragma unroll
    for (int x0 = 0; x0 < kA; x0 += kTurn) {
#pragma unroll
        for (int x = 0; x < kTurn; ++x)
#pragma unroll
            for (int y = 0; y < kB; ++y)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    turn[place(32 * x + 8 * (r / 4) + 4 * (lane / 32) + r % 4, 32 * y + lane % 32)] = acc[x0 + x][y][r];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int64_t i0x = i0 + wi + 32 * x0;
#pragma unroll 1
        for (int r0 = lane / kLanes; r0 < 32 * kTurn; r0 += kAhead * kStepRows) {
            Extras<T> extra[kAhead];
            if (!kColumnsB && p.count == 1 && left > 0)
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (const int64_t i = i0x + r0 + u * kStepRows; i < p.m) extra[u].load(p.e, i, j, left);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int row = r0 + u * kStepRows;
                const int64_t i = i0x + row;
                float z[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) z[c] = turn[place(row, column) + c];
                if (i >= p.m || left <= 0) continue;
                if (p.count > 1) {
                    store_some(p.parts + (t.part * p.m + i) * ((p.n + 7) / 8 * 8) + j, 8, z);
                } else if constexpr (kColumnsB) {                 // dx and dweight have no epilogue
                    Kind::template store<T>(p, i, j, left, z);
                } else {
                    finish8<T>(p.e, i, j, left, bias, extra[u], z);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int kTileM, int kTileN, int kSteps>
constexpr int kTilesPerCu = (kTileM + kTileN) * kSteps > 512 ? 1 : 2;

template <typename T, bool kColumnsA, bool kColumnsB, int kTileM, int kTileN, int kSteps>
__global__ __launch_bounds__(256, (kTilesPerCu<kTileM, kTileN, kSteps>)) void product_kernel(const Product p) {
    product_tile<T, kColumnsA, kColumnsB, kTileM, kTileN, kSteps, OneMatrix>(p);
}

}  // namespace
}  // namespace fsdp_block
