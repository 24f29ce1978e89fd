// Matrix products over two weights that share their input (block_product.h has
// the tiles): a gated feed-forward's forward product, and the gradients of its
// input and of its weights.
#pragma once

#include "block_product.h"
#include "step_saved.h"
#include "step_tile.h"

namespace fsdp_block {
namespace {

// In a forward product n, j and the tiles count the columns of both matrices,
// n = 2 * inner; in the gradients `inner` columns of the first of dz's two parts
// lie before column `split`, where the second begins.
struct PairProduct : Product {
    const void* b2;
    int64_t b2_stride, inner, split;
    // Forward: g and u for the gradient, as values or codes and scales.
    void *gate, *up;
    uint8_t *gate_scales, *up_scales;
    int64_t gate_stride, up_stride, gate_scales_stride, up_scales_stride;
    // The weights' gradients: the second one.
    void* out2;
    int64_t out2_stride;
};

// fp32: runs of 512 k. One sum over k = 7864 is off by 1.6e-6 of the result (2-norm), in runs by
// 4.1e-7; they cost 1 to 3 % (1910 x 1024 x 7864: 551 us, 537 without).
constexpr int kRunSteps = 16;

// Columns of g (or u) in a row of the parts.
__device__ __host__ __forceinline__ int64_t part_columns(int64_t inner) { return (inner + 7) / 8 * 8; }

// f(activation) with the activation as a constant: one choice for many values, so that
// their chains of instructions overlap.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case FSDP_ACT_RELU: return f(std::integral_constant<int, FSDP_ACT_RELU>());
        case FSDP_ACT_SILU: return f(std::integral_constant<int, FSDP_ACT_SILU>());
        case FSDP_ACT_GELU: return f(std::integral_constant<int, FSDP_ACT_GELU>());
        case FSDP_ACT_GELU_TANH: return f(std::integral_constant<int, FSDP_ACT_GELU_TANH>());
        default: return f(std::integral_constant<int, FSDP_ACT_NONE>());
    }
}

// g and u at row i, columns j .. j + 7, of which `left` exist; four lanes (kApart: as in
// group_max) have a row's group of 32 columns, and all of them come here.
template <typename T, bool kApart>
__device__ __forceinline__ void keep8(void* kept, uint8_t* scales, int64_t stride, int64_t scales_stride, int64_t i, int64_t j, int left,
                                      const float (&z)[8]) {
    if (!kept) return;
    if (scales)
        save8<kApart>(z, left, static_cast<int8_t*>(kept) + i * stride + j, scales + i * scales_stride + j / FSDP_STEP_GROUP);
    else if (left > 0)
        store_some(static_cast<T*>(kept) + i * stride + j, left, z);
}
template <typename T, bool kApart = false>
__device__ __forceinline__ void finish_pair(const PairProduct& p, int64_t i, int64_t j, int left, const float (&g)[8], const float (&u)[8]) {
    keep8<T, kApart>(p.gate, p.gate_scales, p.gate_stride, p.gate_scales_stride, i, j, left, g);
    keep8<T, kApart>(p.up, p.up_scales, p.up_stride, p.up_scales_stride, i, j, left, u);
    if (left <= 0) return;
    float out[8];
    with_act(p.e.act, [&](auto act) {
#pragma unroll
        for (int c = 0; c < 8; ++c) out[c] = act_value<sizeof(T) == 4>(g[c], decltype(act)::value) * u[c];
    });
    store_some(static_cast<T*>(p.e.out) + i * p.e.out_stride + j, left, out);
}

// As finish_pair, kApart, of several times eight columns that all exist: kDown rows 16 apart of kAcross
// groups. Without branches of their own, so that their chains of instructions overlap where a SIMD
// has one wave.
template <typename T, int kDown, int kAcross>
__device__ __forceinline__ void finish_whole(const PairProduct& p, int64_t i, int64_t j, const float (&g)[kDown][kAcross][8],
                                             const float (&u)[kDown][kAcross][8]) {
    const auto keep = [&](void* kept, uint8_t* scales, int64_t stride, int64_t scales_stride, const float (&z)[kDown][kAcross][8]) {
        if (!kept) return;
        if (scales) {
            uint32_t byte[kDown][kAcross];
#pragma unroll
            for (int d = 0; d < kDown; ++d)
#pragma unroll
                for (int a = 0; a < kAcross; ++a) {
                    uint32_t most = 0;
#pragma unroll
                    for (int c = 0; c < 8; ++c) most = max(most, __builtin_bit_cast(uint32_t, z[d][a][c]) & 0x7fffffffu);
                    byte[d][a] = scale_byte(group_max<true>(most));
                }
            int8_t* const codes = static_cast<int8_t*>(kept) + i * stride + j;
#pragma unroll
            for (int d = 0; d < kDown; ++d)
#pragma unroll
                for (int a = 0; a < kAcross; ++a)
                    reinterpret_cast<AnyCodes*>(codes + 16 * d * stride + FSDP_STEP_GROUP * a)->v = codes_of(z[d][a], byte[d][a]);
            if ((threadIdx.x & 48) != 0) return;
            uint8_t* const scale = scales + i * scales_stride + j / FSDP_STEP_GROUP;
#pragma unroll
            for (int d = 0; d < kDown; ++d)
#pragma unroll
                for (int a = 0; a < kAcross; ++a) scale[16 * d * scales_stride + a] = uint8_t(byte[d][a]);
        } else {
            T* const at = static_cast<T*>(kept) + i * stride + j;
#pragma unroll
            for (int d = 0; d < kDown; ++d)
#pragma unroll
                for (int a = 0; a < kAcross; ++a) store_some(at + 16 * d * stride + FSDP_STEP_GROUP * a, 8, z[d][a]);
        }
    };
    keep(p.gate, p.gate_scales, p.gate_stride, p.gate_scales_stride, g);
    keep(p.up, p.up_scales, p.up_stride, p.up_scales_stride, u);
    T* const at = static_cast<T*>(p.e.out) + i * p.e.out_stride + j;
    with_act(p.e.act, [&](auto act) {
        float out[kDown][kAcross][8];
#pragma unroll
        for (int d = 0; d < kDown; ++d)
#pragma unroll
            for (int a = 0; a < kAcross; ++a)
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    out[d][a][c] = act_value<sizeof(T) == 4>(g[d][a][c], decltype(act)::value) * u[d][a][c];
#pragma unroll
        for (int d = 0; d < kDown; ++d)
#pragma unroll
            for (int a = 0; a < kAcross; ++a) store_some(at + 16 * d * p.e.out_stride + FSDP_STEP_GROUP * a, 8, out[d][a]);
    });
}

// ------------------------------------------------------------------ forward

// Rows of two matrices: the first half of a tile's from one, the second half from the
// other.  As Operand, by rows.
template <typename T, int kRows>
struct PairRows {
    using One = Operand<T, kRows, false>;
    static constexpr int kBytes = One::kBytes, kLoads = One::kLoads, kUnit = One::kUnit;
    const char* at[2];
    int64_t left[2];
    uint32_t offset[kLoads];
    int k;

    __device__ __forceinline__ PairRows(const PairProduct& p, int64_t first, int64_t k0, int64_t k1) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int u = lane % 8 ^ (wave % 2 * 4 + lane / 16);
        k = u * kUnit;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t stride = h ? p.b2_stride : p.b_stride;
            at[h] = static_cast<const char*>(h ? p.b2 : p.b) + (first * stride + k0) * One::kSize;
            left[h] = (p.inner - 1 - first) * stride * One::kSize + (k1 - k0 + kUnit - 1) / kUnit * 16;
#pragma unroll
            for (int j = 0; j < kLoads / 2; ++j) {
                const int row = (j * 4 + wave) * 8 + lane / 8;
                offset[h * (kLoads / 2) + j] = uint32_t(min(row * stride * One::kSize + u * 16, One::kNowhere));
            }
        }
    }
    __device__ __forceinline__ void load(char* lds, int64_t rest) {
        typedef __attribute__((address_space(3))) void lds_void;
        constexpr uint32_t kMost = 0x7ffffff0u;
        const bool mine = k < rest;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t bytes = rest <= 0 ? 0u : uint32_t(min(left[h], int64_t(kMost)));
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at[h]), 0, int(bytes), 0x00020000);
#pragma unroll
            for (int j = h * (kLoads / 2); j < (h + 1) * (kLoads / 2); ++j)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)(lds + (j * 4 + (threadIdx.x >> 6)) * 1024), 16,
                                                         int(mine ? offset[j] : uint32_t(One::kNowhere)), 0, 0, 0);
            at[h] += 128;
            left[h] -= 128;
        }
    }
};

// The same for step_tile.h.
template <typename T, int kRows>
struct PairStream : Stream<T, kRows, false> {
    using One = Stream<T, kRows, false>;
    static constexpr int kHalf = One::kLoads / 2;
    const char* at2;
    int64_t left2;
    __amdgpu_buffer_rsrc_t from2;
    __device__ __forceinline__ PairStream(const PairProduct& p, int64_t first, int64_t k0, int64_t k1)
        : One(p.b, p.b_stride, first, p.inner, k0, k1) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        this->k = (lane % 8 ^ (wave * 2 + lane / 16 % 2)) * 8;       // as a woven Half reads them
        at2 = static_cast<const char*>(p.b2) + (first * p.b2_stride + k0) * 2;
        left2 = (p.inner - 1 - first) * p.b2_stride * 2 + (k1 - k0 + 7) / 8 * 16;
#pragma unroll
        for (int j = 0; j < kHalf; ++j) {
            this->offset[j] = uint32_t(min(((j * 4 + wave) * 8 + lane / 8) * p.b_stride * 2 + this->k * 2, One::kNowhere));
            this->offset[kHalf + j] = uint32_t(min(((j * 4 + wave) * 8 + lane / 8) * p.b2_stride * 2 + this->k * 2, One::kNowhere));
        }
    }
    __device__ __forceinline__ void next() {
        from2 = this->range(at2, left2);
        at2 += 128;
        left2 -= 128;
        One::next();
    }
    __device__ __forceinline__ void load(char* lds, int j, int own) const {
        typedef __attribute__((address_space(3))) void lds_void;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(j < kHalf ? this->from : from2, (lds_void*)(lds + j * 4096 + own), 16,
                                                 int(this->offset[j]), 0, 0, 0);
    }
};

// out = act(x gate^T) * (x up^T): a wave has the same columns of both products, side
// by side in its registers and in its piece of LDS.
struct GatedForward {
    static constexpr bool kPair = true;
    static constexpr int kRun = kRunSteps;
    template <typename T, int kTileN, bool kColumnsB>
    using B = PairRows<T, kTileN>;
    template <typename T, int kTileN, bool kColumnsB>
    __device__ static __forceinline__ auto operand(const PairProduct& p, int64_t j0, int64_t k0, int64_t k1) {
        return B<T, kTileN, kColumnsB>(p, j0 / 2, k0, k1);
    }
    template <typename T, int kTile, bool kColumnsB>
    using Ring = PairStream<T, kTile>;
    template <typename T, int kTile, bool kColumnsB>
    __device__ static __forceinline__ auto ring_operand(const PairProduct& p, int64_t j0, int64_t k0, int64_t k1) {
        return PairStream<T, kTile>(p, j0 / 2, k0, k1);
    }
    // Eight columns of a row from a ring tile's registers: lanes 16 apart have a group of 32.
    template <typename T>
    __device__ static __forceinline__ void put(const PairProduct& p, int part, int64_t i, int64_t j, const float (&g)[8], const float (&u)[8]) {
        const int left = int(min(p.inner - j, int64_t(8)));
        if (i >= p.m) return;
        if (p.count > 1) {
            store_parts(p, part, i, j, left, g, u);
        } else {
            finish_pair<T, true>(p, i, j, left, g, u);
        }
    }
    template <typename T, int kDown, int kAcross>
    __device__ static __forceinline__ void put_whole(const PairProduct& p, int64_t i, int64_t j, const float (&g)[kDown][kAcross][8],
                                                     const float (&u)[kDown][kAcross][8]) {
        finish_whole<T>(p, i, j, g, u);
    }
    // Whether the tile at row i, columns j (of g) on goes to its places whole.
    __device__ static __forceinline__ bool whole(const PairProduct& p, int64_t i, int64_t j, int tile) {
        return p.count == 1 && i + tile <= p.m && j + tile / 2 <= p.inner;
    }
    __device__ static __forceinline__ void store_parts(const PairProduct& p, int part, int64_t i, int64_t j, int left, const float (&g)[8],
                                                       const float (&u)[8]) {
        float* const at = p.parts + (part * p.m + i) * 2 * part_columns(p.inner) + j;
        if (left <= 0) return;
        store_some(at, 8, g);
        store_some(at + part_columns(p.inner), 8, u);
    }
    // Rows first_i on, columns first_j on of kWide / 2; `pieces` calls back with a piece's
    // first row and how many it has, once they lie in LDS.
    template <typename T, int kWide, typename Place, typename Pieces>
    __device__ static __forceinline__ void finish(const PairProduct& p, int part, const float* turn, Place place, int64_t first_i,
                                                  int64_t first_j, Pieces pieces) {
        constexpr int kHalf = kWide / 2, kLanes = kHalf / 8, kStepRows = 64 / kLanes;
        static_assert(kLanes % 4 == 0);
        const int lane = threadIdx.x & 63, column = lane % kLanes * 8;
        const int64_t j = first_j + column;
        const int left = int(min(p.inner - j, int64_t(8)));
        pieces([&](int first, int rows) {
#pragma unroll 1
            for (int r = lane / kLanes; r < rows; r += kStepRows) {
                const int64_t i = first_i + first + r;
                float g[8], u[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    g[c] = turn[place(r, column) + c];
                    u[c] = turn[place(r, kHalf + column) + c];
                }
                if (i >= p.m) continue;
                if (p.count > 1) store_parts(p, part, i, j, left, g, u);
                else finish_pair<T>(p, i, j, left, g, u);
            }
        });
    }
};

// The parts' sums, in order: a thread takes eight columns of g and of u, a quad a
// group.
template <typename T>
__global__ __launch_bounds__(256) void join_gated_kernel(const PairProduct p) {
    const int64_t wide = part_columns(p.inner), units = (p.inner + 31) / 32 * 4;
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < p.m * units; at += int64_t(gridDim.x) * 256) {
        const int64_t i = at / units, j = at % units * 8;
        const int left = int(min(p.inner - j, int64_t(8)));
        float g[8] = {}, u[8] = {};
        if (left > 0)
            for (int s = 0; s < p.count; ++s) {
                const float* const from = p.parts + (s * p.m + i) * 2 * wide + j;
                const Eight<float> a = load8(from), b = load8(from + wide);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    g[c] += a[c];
                    u[c] += b[c];
                }
            }
        finish_pair<T>(p, i, j, left, g, u);
    }
}

// ------------------------------------------------------------------ gradients

// dx = [dg | du] [gate_weight; up_weight]: k runs over the first matrix's rows, then
// from `split` on, a whole number of steps, over the second's.
template <typename T, int kRows>
struct JoinedColumns : Operand<T, kRows, true> {
    using One = Operand<T, kRows, true>;
    const char* at2;
    int64_t left2, until;            // bytes of the second matrix; k's before it
    __device__ __forceinline__ JoinedColumns(const PairProduct& p, int64_t first, int64_t k0, int64_t k1)
        : One(k0 < p.split ? p.b : p.b2, p.b_stride, first, p.n, k0 < p.split ? k0 : k0 - p.split,
              min(k0 < p.split ? k1 : k1 - p.split, p.inner)) {
        at2 = static_cast<const char*>(p.b2) + first * One::kSize;
        left2 = k1 > p.split ? (min(k1 - p.split, p.inner) - 1) * p.b_stride * One::kSize + (p.n - first + One::kUnit - 1) / One::kUnit * 16 : 0;
        until = k0 < p.split ? p.split - k0 : INT64_MAX;
    }
    __device__ __forceinline__ void load(char* lds, int64_t rest) {
        if (until <= 0) {
            this->at = at2;
            this->left = left2;
            until = INT64_MAX;
        }
        One::load(lds, rest);
        until -= One::kDeep;
    }
};

// The same for step_tile.h.
template <typename T, int kRows>
struct JoinedStream : Stream<T, kRows, true> {
    using One = Stream<T, kRows, true>;
    const char* at2;
    int64_t left2;
    int until;
    __device__ __forceinline__ JoinedStream(const PairProduct& p, int64_t first, int64_t k0, int64_t k1)
        : One(k0 < p.split ? p.b : p.b2, p.b_stride, first, p.n, k0 < p.split ? k0 : k0 - p.split,
              min(k0 < p.split ? k1 : k1 - p.split, p.inner)) {
        at2 = static_cast<const char*>(p.b2) + first * 2;
        left2 = k1 > p.split ? (min(k1 - p.split, p.inner) - 1) * p.b_stride * 2 + (p.n - first + 7) / 8 * 16 : 0;
        until = k0 < p.split ? int(min(p.split - k0, int64_t(INT32_MAX))) : INT32_MAX;
        this->rest = int(k1 - k0);
    }
    __device__ __forceinline__ void next() {
        if (until <= 0) {
            this->at = at2;
            this->left = left2;
            until = INT32_MAX;
        }
        One::next();
        until -= 64;
    }
};

// Rows from p on.
struct RowsOut {
    void* p;
    int64_t stride;
};

// Eight columns of a row to their place.
template <typename Kind>
struct Plain : OneMatrix {
    static constexpr int kRun = kRunSteps;
    template <typename T, int kWide, typename Place, typename Pieces>
    __device__ static __forceinline__ void finish(const PairProduct& p, int part, const float* turn, Place place, int64_t first_i,
                                                  int64_t first_j, Pieces pieces) {
        constexpr int kLanes = kWide / 8, kStepRows = 64 / kLanes;
        const int lane = threadIdx.x & 63, column = lane % kLanes * 8;
        const int64_t j = first_j + column;
        const int left = int(min(p.n - j, int64_t(8)));
        const auto fetch = [&](int r, float (&z)[8]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(turn + place(r, column) + 4 * h);
#pragma unroll
                for (int c = 0; c < 4; ++c) z[4 * h + c] = v[c];
            }
        };
        pieces([&](int first, int rows) {
            // A piece that lies in one output whole: rows together, without branches of their own (the
            // gradient of 1024 x 14336 x 1024 in fp16: 171 us instead of 178).
            if (p.count == 1 && first_j + kWide <= p.n && Kind::whole(p, first_i + first, rows)) {
                constexpr int kMany = 4;
                const RowsOut to = Kind::template out<T>(p, first_i + first);
                T* const at = static_cast<T*>(to.p) + lane / kLanes * to.stride + j;
#pragma unroll 1
                for (int r = 0; r < rows; r += kMany * kStepRows) {
                    float z[kMany][8];
#pragma unroll
                    for (int q = 0; q < kMany; ++q) fetch(r + q * kStepRows + lane / kLanes, z[q]);
#pragma unroll
                    for (int q = 0; q < kMany; ++q) store_some(at + (r + q * kStepRows) * to.stride, 8, z[q]);
                }
                return;
            }
#pragma unroll 4
            for (int r = lane / kLanes; r < rows; r += kStepRows) {
                const int64_t i = first_i + first + r;
                float z[8];
                fetch(r, z);
                if (i >= p.m || left <= 0) continue;
                if (p.count > 1) store_some(p.parts + (part * p.m + i) * ((p.n + 7) / 8 * 8) + j, 8, z);
                else Kind::template store<T>(p, i, j, left, z);
            }
        });
    }
};

struct PairInput : Plain<PairInput> {
    __device__ static __forceinline__ bool whole(const PairProduct& p, int64_t i, int rows) { return i + rows <= p.m; }
    template <typename T>
    __device__ static __forceinline__ RowsOut out(const PairProduct& p, int64_t i) {
        return {static_cast<T*>(p.e.out) + i * p.e.out_stride, p.e.out_stride};
    }
    template <typename T, int kTileN, bool kColumnsB>
    using B = JoinedColumns<T, kTileN>;
    template <typename T, int kTileN, bool kColumnsB>
    __device__ static __forceinline__ auto operand(const PairProduct& p, int64_t j0, int64_t k0, int64_t k1) {
        return B<T, kTileN, kColumnsB>(p, j0, k0, k1);
    }
    template <typename T, int kTile, bool kColumnsB>
    using Ring = JoinedStream<T, kTile>;
    template <typename T, int kTile, bool kColumnsB>
    __device__ static __forceinline__ auto ring_operand(const PairProduct& p, int64_t j0, int64_t k0, int64_t k1) {
        return JoinedStream<T, kTile>(p, j0, k0, k1);
    }
};

// [dgate_weight; dup_weight] = [dg | du]^T x: rows from `split` on are the second's.
struct PairWeights : Plain<PairWeights> {
    __device__ static __forceinline__ bool whole(const PairProduct& p, int64_t i, int rows) {
        return i + rows <= p.inner || (i >= p.split && i + rows <= p.m);
    }
    template <typename T>
    __device__ static __forceinline__ RowsOut out(const PairProduct& p, int64_t i) {
        if (i < p.inner) return {static_cast<T*>(p.e.out) + i * p.e.out_stride, p.e.out_stride};
        return {static_cast<T*>(p.out2) + (i - p.split) * p.out2_stride, p.out2_stride};
    }
    template <typename T, int kTile, bool kColumnsB>
    using Ring = Stream<T, kTile, true>;
    template <typename T, int kTile, bool kColumnsB>
    __device__ static __forceinline__ auto ring_operand(const PairProduct& p, int64_t j0, int64_t k0, int64_t k1) {
        return Stream<T, kTile, true>(p.b, p.b_stride, j0, p.n, k0, k1);
    }
    template <typename T>
    __device__ static __forceinline__ void store(const PairProduct& p, int64_t i, int64_t j, int left, const float (&z)[8]) {
        if (i < p.inner) store_some(static_cast<T*>(p.e.out) + i * p.e.out_stride + j, left, z);
        else if (i >= p.split) store_some(static_cast<T*>(p.out2) + (i - p.split) * p.out2_stride + j, left, z);
    }
};

template <typename T, typename Kind>
__global__ __launch_bounds__(256) void join_pair_kernel(const PairProduct p) {
    const int64_t units = (p.n + 7) / 8, stride = units * 8;
    for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < p.m * units; u += int64_t(gridDim.x) * 256) {
        const int64_t i = u / units, j = u % units * 8;
        float z[8] = {};
        for (int s = 0; s < p.count; ++s) {
            const Eight<float> v = load8(p.parts + (s * p.m + i) * stride + j);
#pragma unroll
            for (int c = 0; c < 8; ++c) z[c] += v[c];
        }
        Kind::template store<T>(p, i, j, int(min(p.n - j, int64_t(8))), z);
    }
}

template <typename T, typename Kind, int kTileM, int kTileN, int kSteps>
__global__ __launch_bounds__(256, (kTilesPerCu<kTileM, kTileN, kSteps>)) void pair_kernel(const PairProduct p) {
    constexpr bool kForward = std::is_same<Kind, GatedForward>::value, kWeights = std::is_same<Kind, PairWeights>::value;
    product_tile<T, kWeights, !kForward, kTileM, kTileN, kSteps, Kind>(p);
}

// Tiles of step_tile.h; with kRing = 5 of 128 x 128 two lie on a CU.
template <typename T, typename Kind, int kTile, int kRing>
__global__ __launch_bounds__(256, (kTile * kRing > 640 ? 1 : 2)) void ring_kernel(const PairProduct p) {
    constexpr bool kForward = std::is_same<Kind, GatedForward>::value, kWeights = std::is_same<Kind, PairWeights>::value;
    ring_tile<T, kWeights, !kForward, kTile, kRing, Kind>(p);
}

}  // namespace
}  // namespace fsdp_block
