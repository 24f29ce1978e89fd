// The matrix product with bias, activation, factor and residual in its
// epilogue, and its gradient (include/fsdp_block.h).
//
// All three products (x W^T, dz W, dz^T x) are out[i][j] = sum_k A[i][k] B[j][k]
// with A and B row-major in i / j ("rows") or in k ("columns").

#include "block_device.h"
#include "block_host.h"
#include "block_join.h"

#include <algorithm>

namespace fsdp_block {
namespace {

// ------------------------------------------------------------------ elementwise

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }

// act(z); 1 + tanh(u) is 2 sigmoid(2u).
__device__ __forceinline__ float act_value(float z, int act) {
    switch (act) {
        case FSDP_ACT_RELU: return z != z ? z : fmaxf(z, 0.f);
        case FSDP_ACT_SILU: return z * sigmoid(z);
        case FSDP_ACT_GELU: return 0.5f * z * erfcf(-0.70710678118654752f * z);
        case FSDP_ACT_GELU_TANH: return z * sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z));
        default: return z;
    }
}

__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
        case FSDP_ACT_RELU: return z != z ? z : z > 0.f ? 1.f : 0.f;
        case FSDP_ACT_SILU: {
            const float q = sigmoid(z);
            return q * (1.f + z * (1.f - q));
        }
        case FSDP_ACT_GELU:
            return 0.5f * erfcf(-0.70710678118654752f * z) + z * (0.39894228040143268f * expf(-0.5f * z * z));
        case FSDP_ACT_GELU_TANH: {
            const float q = sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z));
            return q + z * (q * (1.f - q)) * (1.5957691216057308f * (1.f + 0.134145f * z * z));
        }
        default: return 1.f;
    }
}

// ------------------------------------------------------------------ epilogue

struct Epilogue {
    const void *bias, *times, *residual;
    void *pre, *out;
    int64_t times_stride, residual_stride, pre_stride, out_stride;
    int act;
};

// z -> out at row i, column j; `z` is the product, without the bias.
template <typename T>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t i, int64_t j, float z) {
    if (e.bias) z += float(static_cast<const T*>(e.bias)[j]);
    if (e.pre) static_cast<T*>(e.pre)[i * e.pre_stride + j] = T(z);
    z = act_value(z, e.act);
    if (e.times) z *= float(static_cast<const T*>(e.times)[i * e.times_stride + j]);
    if (e.residual) z += float(static_cast<const T*>(e.residual)[i * e.residual_stride + j]);
    static_cast<T*>(e.out)[i * e.out_stride + j] = T(z);
}

// ------------------------------------------------------------------ product

struct Product {
    const void *a, *b;
    int64_t a_stride, b_stride;
    int64_t m, n, k;                 // out [m, n]
    Epilogue e;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

// 16 bytes of A rows and of B rows per lane -> a 16 x 16 tile.  Lane l holds
// row l % 16 of both and the (l / 16)-th 16 bytes of a 64-byte run of k; the
// tile's element r of lane l is at A row 4 (l / 16) + r, B row l % 16.
__device__ __forceinline__ f32x4 mma(Eight<bf16> a, Eight<bf16> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(Eight<f16> a, Eight<f16> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// The 16 bytes that a load and a lane of a matrix instruction take.
template <typename T>
struct Unit {
    static constexpr int n = 16 / int(sizeof(T));
    typedef T type __attribute__((ext_vector_type(n)));
    struct __attribute__((packed, aligned(sizeof(T)))) any {
        type v;
    };
};

// A 128 x 128 tile of out in 256 threads, from operands of any alignment,
// stride and size: the form for what the aligned one does not take.
constexpr int kAnyTile = 128;

// Loads two units of a 128-row, 64-byte operand tile: of rows first + .., k from
// k0.  kColumns: the operand lies k-major, a unit is n rows at one k.
template <typename T, bool kColumns>
__device__ __forceinline__ void load_any(const T* p, int64_t stride, int64_t first, int64_t rows, int64_t k0, int64_t k,
                                         typename Unit<T>::type (&out)[2]) {
    constexpr int n = Unit<T>::n, kDeep = 4 * n;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int c = int(threadIdx.x) + 256 * u;
        const int64_t i = first + (kColumns ? c % (kAnyTile / n) * n : c / 4);
        const int64_t j = k0 + (kColumns ? c / (kAnyTile / n) : c % 4 * n);
        static_assert(kAnyTile / n * kDeep == 512, "two units per thread");
        const int64_t left = kColumns ? (j < k ? rows - i : 0) : (i < rows ? k - j : 0);
        const T* at = kColumns ? p + j * stride + i : p + i * stride + j;
        if (left >= n) {
            out[u] = reinterpret_cast<const typename Unit<T>::any*>(at)->v;
        } else {
#pragma unroll
            for (int e = 0; e < n; ++e) out[u][e] = e < left ? at[e] : T(0.f);
        }
    }
}

template <typename T>
using AnyTile = T[kAnyTile][5 * Unit<T>::n];     // rows of 64 bytes of k, padded by 16

template <typename T, bool kColumns>
__device__ __forceinline__ void keep_any(AnyTile<T>& tile, const typename Unit<T>::type (&in)[2]) {
    constexpr int n = Unit<T>::n;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int c = int(threadIdx.x) + 256 * u;
        if constexpr (kColumns) {
#pragma unroll
            for (int e = 0; e < n; ++e) tile[c % (kAnyTile / n) * n + e][c / (kAnyTile / n)] = in[u][e];
        } else {
            *reinterpret_cast<typename Unit<T>::type*>(&tile[c / 4][c % 4 * n]) = in[u];
        }
    }
}

template <typename T, bool kColumnsA, bool kColumnsB>
__global__ __launch_bounds__(256) void product_any_kernel(const Product p) {
    constexpr int n = Unit<T>::n, kDeep = 4 * n;
    using U = typename Unit<T>::type;
    __shared__ __attribute__((aligned(16))) AnyTile<T> ta, tb;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wi = wave / 2 * 64, wj = wave % 2 * 64;
    const int64_t tiles_n = (p.n + kAnyTile - 1) / kAnyTile;
    const int64_t i0 = blockIdx.x / tiles_n * kAnyTile, j0 = blockIdx.x % tiles_n * kAnyTile;
    const T* a = static_cast<const T*>(p.a);
    const T* b = static_cast<const T*>(p.b);
    f32x4 acc[4][4] = {};            // [A tile][B tile]
    U ra[2], rb[2];
    load_any<T, kColumnsA>(a, p.a_stride, i0, p.m, 0, p.k, ra);
    load_any<T, kColumnsB>(b, p.b_stride, j0, p.n, 0, p.k, rb);
    for (int64_t k = 0; k < p.k; k += kDeep) {
        __syncthreads();
        keep_any<T, kColumnsA>(ta, ra);
        keep_any<T, kColumnsB>(tb, rb);
        __syncthreads();
        if (k + kDeep < p.k) {
            load_any<T, kColumnsA>(a, p.a_stride, i0, p.m, k + kDeep, p.k, ra);
            load_any<T, kColumnsB>(b, p.b_stride, j0, p.n, k + kDeep, p.k, rb);
        }
        U fa[4], fb[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            fa[x] = *reinterpret_cast<const U*>(&ta[wi + 16 * x + lane % 16][lane / 16 * n]);
            fb[x] = *reinterpret_cast<const U*>(&tb[wj + 16 * x + lane % 16][lane / 16 * n]);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[x][y] = mma(fa[x], fb[y], acc[x][y]);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t i = i0 + wi + 16 * x + lane / 16 * 4 + r, j = j0 + wj + 16 * y + lane % 16;
                if (i < p.m && j < p.n) finish<T>(p.e, i, j, acc[x][y][r]);
            }
}

// ------------------------------------------------------------------ dz

struct SlopeArgs {
    const void *dout, *pre, *times;
    void *dz, *dtimes;
    float* part;                     // [row parts, n] sums of dz, or NULL
    int64_t dout_stride, pre_stride, times_stride, dz_stride, dtimes_stride;
    int64_t m, n, part_rows;
    int act;
};

// A workgroup takes 512 columns, eight per lane, of part_rows rows, one row per
// wave at a time.
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a) {
    __shared__ float sums[4][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = int64_t(blockIdx.x) * 512 + lane * 8;
    const int left = int(min(a.n - j, int64_t(8)));
    const int64_t hi = min((int64_t(blockIdx.y) + 1) * a.part_rows, a.m);
    float sum[8] = {};
    if (left > 0)
        for (int64_t i = int64_t(blockIdx.y) * a.part_rows + wave; i < hi; i += 4) {
            const Eight<T> d = load_some(static_cast<const T*>(a.dout) + i * a.dout_stride + j, left);
            Eight<T> z, f;
            if (a.pre) z = load_some(static_cast<const T*>(a.pre) + i * a.pre_stride + j, left);
            if (a.times) f = load_some(static_cast<const T*>(a.times) + i * a.times_stride + j, left);
            float dz[8];
            if (a.dtimes) {
#pragma unroll
                for (int e = 0; e < 8; ++e) dz[e] = float(d[e]) * act_value(float(z[e]), a.act);
                store_some(static_cast<T*>(a.dtimes) + i * a.dtimes_stride + j, left, dz);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dz[e] = float(d[e]);
                if (a.times) dz[e] *= float(f[e]);
                if (a.act != FSDP_ACT_NONE) dz[e] *= act_slope(float(z[e]), a.act);
                sum[e] += dz[e];
            }
            if (a.dz) store_some(static_cast<T*>(a.dz) + i * a.dz_stride + j, left, dz);
        }
    if (!a.part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][lane * 8 + e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < 512; c += 256) {
        const int64_t column = int64_t(blockIdx.x) * 512 + c;
        if (column < a.n) a.part[blockIdx.y * a.n + column] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    }
}


// ------------------------------------------------------------------ host side

template <typename F>
fsdp_status with_type(fsdp_dtype dtype, F f) {
    return dtype == FSDP_DTYPE_BF16 ? f(bf16(0.f)) : dtype == FSDP_DTYPE_F16 ? f(f16(0.f)) : f(0.f);
}

// One product.  kColumns*: the operand lies k-major.
template <bool kColumnsA, bool kColumnsB>
fsdp_status product(const Product& p, fsdp_dtype dtype, hipStream_t stream) {
    if (p.m == 0 || p.n == 0) return FSDP_OK;
    return with_type(dtype, [&](auto type) {
        const int64_t tiles = ceil_div(p.m, kAnyTile) * ceil_div(p.n, kAnyTile);
        return launch(product_any_kernel<decltype(type), kColumnsA, kColumnsB>, p, dim3(unsigned(tiles)), 256, stream);
    });
}

fsdp_status check_sizes(int64_t m, int64_t n, int64_t k, fsdp_dtype dtype, fsdp_activation act) {
    if (m < 0 || n < 0 || k < 1) return fail(FSDP_ERR_INVALID, "m and n must not be negative, k must be at least 1");
    if (!known_dtype(dtype)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (act < FSDP_ACT_NONE || act > FSDP_ACT_GELU_TANH) return fail(FSDP_ERR_INVALID, "unknown activation");
    // Row and column counts travel as 32-bit values in the kernels, tiles as a launch's workgroups.
    if (m > INT32_MAX / 2 || n > INT32_MAX / 2 || k > INT32_MAX / 2) return fail(FSDP_ERR_OVERFLOW, "a size is above 2^30");
    const int64_t most = int64_t(1) << 22;
    if (ceil_div(m, kAnyTile) * ceil_div(n, kAnyTile) > most || ceil_div(m, kAnyTile) * ceil_div(k, kAnyTile) > most ||
        ceil_div(n, kAnyTile) * ceil_div(k, kAnyTile) > most)
        return fail(FSDP_ERR_OVERFLOW, "a product has too many tiles");
    return FSDP_OK;
}

fsdp_status check_linear(const fsdp_linear_args& a) {
    const fsdp_status st = check_sizes(a.m, a.n, a.k, a.dtype, a.activation);
    if (st != FSDP_OK) return st;
    Checked c;
    c.add("x", a.x, a.m, a.k, a.x_stride, a.dtype, a.n > 0);
    c.add("weight", a.weight, a.n, a.k, a.weight_stride, a.dtype, a.m > 0);
    c.add_vector("bias", a.bias, a.n, a.dtype, false);
    c.add("times", a.times, a.m, a.n, a.times_stride, a.dtype, false);
    c.add("residual", a.residual, a.m, a.n, a.residual_stride, a.dtype, false);
    c.add("pre", a.pre, a.m, a.n, a.pre_stride, a.dtype, false, true);
    c.add("out", a.out, a.m, a.n, a.out_stride, a.dtype, true, true, a.times, a.residual);
    return c.done();
}

fsdp_status check_grad(const fsdp_linear_grad_args& a) {
    const fsdp_status st = check_sizes(a.m, a.n, a.k, a.dtype, a.activation);
    if (st != FSDP_OK) return st;
    const bool any = a.dx || a.dweight || a.dbias || a.dtimes;
    const bool slopes = a.dx || a.dweight || a.dbias;
    if (a.dtimes && !a.times && a.m > 0) return fail(FSDP_ERR_INVALID, "dtimes needs times");
    Checked c;
    c.add("dout", a.dout, a.m, a.n, a.dout_stride, a.dtype, any);
    c.add("x", a.x, a.m, a.k, a.x_stride, a.dtype, a.dweight && a.n > 0);
    c.add("weight", a.weight, a.n, a.k, a.weight_stride, a.dtype, a.dx && a.m > 0);
    c.add("pre", a.pre, a.m, a.n, a.pre_stride, a.dtype, a.dtimes || (slopes && a.activation != FSDP_ACT_NONE));
    c.add("times", a.times, a.m, a.n, a.times_stride, a.dtype, false);
    c.add("dx", a.dx, a.m, a.k, a.dx_stride, a.dtype, false, true);
    c.add("dweight", a.dweight, a.n, a.k, a.dweight_stride, a.dtype, false, true);
    c.add_vector("dbias", a.dbias, a.n, a.dtype, false, true);
    c.add("dtimes", a.dtimes, a.m, a.n, a.dtimes_stride, a.dtype, false, true, a.times);
    return c.done();
}

// What a gradient needs besides its outputs.
struct GradParts {
    bool slopes = false;             // dz is not dout
    int64_t parts = 0, part_rows = 1;            // row parts of dbias
    int64_t dz = -1, dbias = -1;     // byte offsets
    int64_t bytes = 0;
};

GradParts parts_of(const fsdp_linear_grad_args& a, int cus) {
    GradParts g;
    if (a.m == 0 || a.n == 0) return g;
    g.slopes = a.times || a.activation != FSDP_ACT_NONE;
    const int64_t columns = ceil_div(a.n, 512);
    g.part_rows = std::max<int64_t>(4, round_up(ceil_div(a.m * columns, 8 * int64_t(cus)), 4));
    g.parts = ceil_div(a.m, g.part_rows);
    if (g.slopes && (a.dx || a.dweight)) {
        g.dz = g.bytes;
        g.bytes += round_up(a.m * round_up(a.n, 8) * elem_bytes(a.dtype), 256);
    }
    if (a.dbias) {
        g.dbias = g.bytes;
        g.bytes += round_up(g.parts * a.n * 4, 256);
    }
    return g;
}

}  // namespace
}  // namespace fsdp_block

using namespace fsdp_block;

extern "C" fsdp_status fsdp_block_linear_workspace(const fsdp_linear_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    const fsdp_status st = check_linear(*args);
    if (st != FSDP_OK) return st;
    *bytes = 0;
    return FSDP_OK;
}

extern "C" fsdp_status fsdp_block_linear(const fsdp_linear_args* args, void* workspace, int64_t workspace_bytes,
                                         hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_linear_args& a = *args;
    const fsdp_status st = check_linear(a);
    if (st != FSDP_OK) return st;
    const Product p{a.x, a.weight, a.x_stride, a.weight_stride, a.m, a.n, a.k,
                    {a.bias, a.times, a.residual, a.pre, a.out, a.times_stride, a.residual_stride, a.pre_stride,
                     a.out_stride, a.activation}};
    return product<false, false>(p, a.dtype, stream);
}

extern "C" fsdp_status fsdp_block_linear_grad_workspace(const fsdp_linear_grad_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    fsdp_status st = check_grad(*args);
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    *bytes = parts_of(*args, cus).bytes;
    return FSDP_OK;
}

extern "C" fsdp_status fsdp_block_linear_grad(const fsdp_linear_grad_args* args, void* workspace, int64_t workspace_bytes,
                                              hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_linear_grad_args& a = *args;
    fsdp_status st = check_grad(a);
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    const GradParts g = parts_of(a, cus);
    if ((st = check_workspace(workspace, workspace_bytes, g.bytes)) != FSDP_OK) return st;
    char* const ws = static_cast<char*>(workspace);
    const void* dz = a.dout;
    int64_t dz_stride = a.dout_stride;
    if (g.dz >= 0) {
        dz = ws + g.dz;
        dz_stride = round_up(a.n, 8);
    }
    float* const part = g.dbias < 0 ? nullptr : reinterpret_cast<float*>(ws + g.dbias);
    if (a.m > 0 && a.n > 0 && (g.dz >= 0 || part || a.dtimes)) {
        const SlopeArgs s{a.dout, a.pre, a.times, g.dz >= 0 ? ws + g.dz : nullptr, a.dtimes, part, a.dout_stride,
                          a.pre_stride, a.times_stride, dz_stride, a.dtimes_stride, a.m, a.n, g.part_rows, a.activation};
        const dim3 grid(unsigned(ceil_div(a.n, 512)), unsigned(g.parts));
        st = with_type(a.dtype, [&](auto type) { return launch(slope_kernel<decltype(type)>, s, grid, 256, stream); });
        if (st != FSDP_OK) return st;
    }
    Join j(int(a.n));
    j.add(a.dbias, part, g.parts, a.dbias ? 1 : 0, a.dtype);
    if ((st = j.run(a.dtype, stream)) != FSDP_OK) return st;
    if (a.dx) {
        const Product p{dz, a.weight, dz_stride, a.weight_stride, a.m, a.k, a.n,
                        {nullptr, nullptr, nullptr, nullptr, a.dx, 0, 0, 0, a.dx_stride, FSDP_ACT_NONE}};
        if ((st = product<false, true>(p, a.dtype, stream)) != FSDP_OK) return st;
    }
    if (a.dweight) {
        const Product p{dz, a.x, dz_stride, a.x_stride, a.n, a.k, a.m,
                        {nullptr, nullptr, nullptr, nullptr, a.dweight, 0, 0, 0, a.dweight_stride, FSDP_ACT_NONE}};
        st = product<true, true>(p, a.dtype, stream);
    }
    return st;
}
