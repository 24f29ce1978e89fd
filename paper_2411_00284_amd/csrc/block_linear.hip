// The matrix product with bias, activation, factor and residual in its
// epilogue, and its gradient (include/fsdp_block.h).
//
// A product takes one of these forms:
//   * product_kernel (block_product.h): operands on the 16-byte grid, in tiles of
//     256 x 256, 64 x 64 (16 bits only), 128 x 128 or 64 x 128.  Operands off the grid
//     are laid on it by a copy into the workspace first.
//   * row_kernel: at most four rows of x, at any address.
// With few tiles the sum over k is cut into parts, which join_parts_kernel joins
// in order; with many, a last round of few tiles is a launch of its own.

#include "block_cut.h"
#include "block_join.h"
#include "block_lay.h"
#include "block_product.h"

#include <algorithm>

namespace fsdp_block {
namespace {

// ------------------------------------------------------------------ few rows

// x W^T of at most kRows rows of x: a wave takes kOut rows of W, eight elements
// per lane at a time, and reads W once, past the caches (16 bits: 22.6 instead of
// 24.4 us at 1 x 14336 x 4096, 5.2 TB/s; fp32 elements are half a line a load and
// stay); x comes from cache, the more of it per row of W the more rows there are.
template <typename T, int kRows>
constexpr int kRowOut = kRows > 2 ? 4 : 2;

template <typename T, int kRows>
__global__ __launch_bounds__(256) void row_kernel(const Product p) {
    constexpr int kOut = kRowOut<T, kRows>, kTogether = 8 / kOut;
    const int lane = threadIdx.x & 63;
    const int64_t j0 = (int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6)) * kOut;
    if (j0 >= p.n) return;
    const T* w[kOut];
#pragma unroll
    for (int o = 0; o < kOut; ++o) w[o] = static_cast<const T*>(p.b) + min(j0 + o, p.n - 1) * p.b_stride;
    const T* x = static_cast<const T*>(p.a);
    float sum[kOut][kRows] = {};
    const auto add = [&](int64_t k, int n) {
        Eight<T> v[kOut];
#pragma unroll
        for (int o = 0; o < kOut; ++o) v[o] = n == 8 && sizeof(T) == 2 ? load8_once(w[o] + k) : load_some(w[o] + k, n);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const Eight<T> u = load_some(x + min(int64_t(i), p.m - 1) * p.a_stride + k, n);
#pragma unroll
            for (int o = 0; o < kOut; ++o)
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[o][i] += float(v[o][c]) * float(u[c]);
        }
    };
    int64_t k = lane * 8;
#pragma unroll kTogether
    for (; k + 8 <= p.k; k += 512) add(k, 8);
    if (k < p.k) add(k, int(p.k - k));
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int i = 0; i < kRows; ++i) sum[o][i] = wave_sum(sum[o][i]);
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (lane == i && lane < p.m)
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                float z[8] = {sum[o][i]};
                if (j0 + o < p.n) finish8<T>(p.e, i, j0 + o, 1, z);
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
// wave at a time (two or four at a time: 5 to 10 % slower).  Bound by HBM: three
// inputs and dtimes of 4096 x 14336 in bf16, with the sums, take 92 us (5.1 TB/s).
//
// dz is rounded to the type here, because the matrix instructions take factors of
// 16 bits.  That is a rounding as large as the results' own: against 64 bits dx and
// dweight of 4096 x 4096 -> 14336 are off by 2.3e-3 (2-norm, bf16) where the results'
// rounding alone gives 1.7e-3.  Two 16-bit parts of dz would take it away for twice the
// matrix work, which is nine tenths of the call.
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a) {
    __shared__ float sums[4][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = int64_t(blockIdx.x) * 512 + lane * 8;
    const int left = int(min(a.n - j, int64_t(8)));
    const int64_t hi = min((int64_t(blockIdx.y) + 1) * a.part_rows, a.m);
    float sum[8] = {};
    // Read once, past the caches (16 bits: 92 instead of 103 us; see row_kernel for fp32).
    const auto get = [&](const void* p, int64_t stride, int64_t i) {
        const T* at = static_cast<const T*>(p) + i * stride + j;
        return left == 8 && sizeof(T) == 2 ? load8_once(at) : load_some(at, left);
    };
    if (left > 0)
        for (int64_t i = int64_t(blockIdx.y) * a.part_rows + wave; i < hi; i += 4) {
            const Eight<T> d = get(a.dout, a.dout_stride, i);
            Eight<T> z, f;
            if (a.pre) z = get(a.pre, a.pre_stride, i);
            if (a.times) f = get(a.times, a.times_stride, i);
            float dz[8], df[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dz[e] = float(d[e]);
                float value = 1.f, slope = 1.f;
                if (a.pre) act_both<sizeof(T) == 4>(float(z[e]), a.act, value, slope);
                df[e] = dz[e] * value;
                if (a.times) dz[e] *= float(f[e]);
                if (a.act != FSDP_ACT_NONE) dz[e] *= slope;
                sum[e] += dz[e];
            }
            if (a.dtimes) store_some(static_cast<T*>(a.dtimes) + i * a.dtimes_stride + j, left, df);
            // dz's rows are the workspace's: whole units, zeros after the columns (load_some gave zeros).
            if (a.dz) store_some(static_cast<T*>(a.dz) + i * a.dz_stride + j, 8, dz);
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

// Adds a product's needs to those of `bytes`.
Cut plan(const Shape& s, const Source& a, const Source& b, int cus, int64_t bytes) {
    Cut c = choose(s, cus, linear_forms(s.dtype));
    c.bytes = bytes;
    if (!c.form || s.m == 0 || s.n == 0 || s.k == 0) return c;
    const auto take = [&](int64_t n) {
        const int64_t at = c.bytes;
        c.bytes += round_up(n, 256);
        return at;
    };
    const int size = elem_bytes(s.dtype);
    if (!on_grid(a, s.dtype)) c.pad_a = take(a.rows * lined(a.cols, s.dtype) * size);
    if (!on_grid(b, s.dtype)) c.pad_b = take(b.rows * lined(b.cols, s.dtype) * size);
    if (c.count > 1) c.parts = take(int64_t(c.count) * s.m * round_up(s.n, 8) * 4);
    return c;
}

template <bool kColumnsA, bool kColumnsB>
fsdp_status launch_tiles(const Product& p, const Form& f, fsdp_dtype dtype, hipStream_t stream) {
    const dim3 grid(unsigned(ceil_div(p.m - p.first_i, f.tile_m) * ceil_div(p.n - p.first_j, f.tile_n) * p.count));
    if (dtype == FSDP_DTYPE_F32)
        return f.tile_m == 128 ? launch(product_kernel<float, kColumnsA, kColumnsB, 128, 128, 2>, p, grid, 256, stream)
                               : launch(product_kernel<float, kColumnsA, kColumnsB, 64, 128, 4>, p, grid, 256, stream);
    const auto of = [&](auto type) {
        using T = decltype(type);
        if (f.tile_m == 256) return launch(product_kernel<T, kColumnsA, kColumnsB, 256, 256, 2>, p, grid, 256, stream);
        if (f.tile_n == 64) return launch(product_kernel<T, kColumnsA, kColumnsB, 64, 64, 8>, p, grid, 256, stream);
        if (f.tile_m == 64) return launch(product_kernel<T, kColumnsA, kColumnsB, 64, 128, 4>, p, grid, 256, stream);
        return f.steps == 2 ? launch(product_kernel<T, kColumnsA, kColumnsB, 128, 128, 2>, p, grid, 256, stream)
                            : launch(product_kernel<T, kColumnsA, kColumnsB, 128, 128, 4>, p, grid, 256, stream);
    };
    return dtype == FSDP_DTYPE_BF16 ? of(bf16(0.f)) : of(f16(0.f));
}

// One product, as `c` says.
fsdp_status run_product(const Shape& s, const Source& a, const Source& b, const Epilogue& e, const Cut& c, char* ws,
                        hipStream_t stream) {
    if (s.m == 0 || s.n == 0) return FSDP_OK;
    Product p{a.p, b.p, a.stride, b.stride, s.m, s.n, s.k, e, nullptr, s.k, 1, 0, 0};
    if (!c.form) {
        return with_type(s.dtype, [&](auto type) {
            using T = decltype(type);
            const auto rows = [&](auto count) {
                constexpr int kRows = decltype(count)::value;
                const dim3 grid(unsigned(ceil_div(s.n, 4 * kRowOut<T, kRows>)));
                return launch(row_kernel<T, kRows>, p, grid, 256, stream);
            };
            return s.m == 1   ? rows(std::integral_constant<int, 1>())
                   : s.m == 2 ? rows(std::integral_constant<int, 2>())
                              : rows(std::integral_constant<int, 4>());
        });
    }
    fsdp_status st;
    Pads<2> pads;
    const auto lay = [&](const Source& o, int64_t at, const void** to, int64_t* stride) {
        if (at < 0) return;
        pads.add(o, s.dtype, ws + at);
        *to = ws + at;
        *stride = lined(o.cols, s.dtype);
    };
    lay(a, c.pad_a, &p.a, &p.a_stride);
    lay(b, c.pad_b, &p.b, &p.b_stride);
    if ((st = pads.run(stream)) != FSDP_OK) return st;
    p.part_k = c.part_k;
    p.count = c.count;
    p.parts = c.parts < 0 ? nullptr : reinterpret_cast<float*>(ws + c.parts);
    const auto tiles = [&](const Form& f) {
        return s.columns_a ? launch_tiles<true, true>(p, f, s.dtype, stream)
               : s.columns_b ? launch_tiles<false, true>(p, f, s.dtype, stream)
                             : launch_tiles<false, false>(p, f, s.dtype, stream);
    };
    if (c.rest) {
        (c.rest_rows ? p.m : p.n) = c.rest_at;
        if ((st = tiles(*c.form)) != FSDP_OK) return st;
        p.m = s.m;
        p.n = s.n;
        (c.rest_rows ? p.first_i : p.first_j) = c.rest_at;
        return tiles(*c.rest);
    }
    if ((st = tiles(*c.form)) != FSDP_OK || c.count == 1) return st;
    const dim3 grid(unsigned(std::min<int64_t>(ceil_div(s.m * ceil_div(s.n, 8), 256), 1 << 13)));
    return with_type(s.dtype, [&](auto type) { return launch(join_parts_kernel<decltype(type)>, p, grid, 256, stream); });
}

fsdp_status check_sizes(int64_t m, int64_t n, int64_t k, fsdp_dtype dtype, fsdp_activation act) {
    if (m < 0 || n < 0 || k < 1) return fail(FSDP_ERR_INVALID, "m and n must not be negative, k must be at least 1");
    if (!known_dtype(dtype)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (act < FSDP_ACT_NONE || act > FSDP_ACT_GELU_TANH) return fail(FSDP_ERR_INVALID, "unknown activation");
    // Row and column counts travel as 32-bit values in the kernels, tiles as a launch's workgroups.
    if (m > INT32_MAX / 2 || n > INT32_MAX / 2 || k > INT32_MAX / 2) return fail(FSDP_ERR_OVERFLOW, "a size is 2^30 or more");
    const int64_t most = int64_t(1) << 22;
    if (ceil_div(m, 64) * ceil_div(n, 64) > most || ceil_div(m, 64) * ceil_div(k, 64) > most ||
        ceil_div(n, 64) * ceil_div(k, 64) > most)
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
    c.add_in_place("times", a.times, a.m, a.n, a.times_stride, a.dtype, false);
    c.add_in_place("residual", a.residual, a.m, a.n, a.residual_stride, a.dtype, false);
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
    c.add_in_place("dout", a.dout, a.m, a.n, a.dout_stride, a.dtype, any);
    c.add("x", a.x, a.m, a.k, a.x_stride, a.dtype, a.dweight && a.n > 0);
    c.add("weight", a.weight, a.n, a.k, a.weight_stride, a.dtype, a.dx && a.m > 0);
    c.add_in_place("pre", a.pre, a.m, a.n, a.pre_stride, a.dtype, a.dtimes || (slopes && a.activation != FSDP_ACT_NONE));
    c.add_in_place("times", a.times, a.m, a.n, a.times_stride, a.dtype, false);
    c.add("dx", a.dx, a.m, a.k, a.dx_stride, a.dtype, false, true);
    c.add("dweight", a.dweight, a.n, a.k, a.dweight_stride, a.dtype, false, true);
    c.add_vector("dbias", a.dbias, a.n, a.dtype, false, true);
    c.add("dtimes", a.dtimes, a.m, a.n, a.dtimes_stride, a.dtype, false, true, a.times);
    return c.done();
}

int64_t row_stride(int64_t rows, int64_t cols, int64_t stride) { return rows > 1 ? stride : round_up(cols, 8); }

// The operands of the three products.
Source forward_x(const fsdp_linear_args& a) { return {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false}; }
Source forward_w(const fsdp_linear_args& a) { return {a.weight, a.n, a.k, row_stride(a.n, a.k, a.weight_stride), false}; }
Shape forward_shape(const fsdp_linear_args& a) {
    return {a.m, a.n, a.k, a.dtype, false, false, laid_stride(forward_x(a), a.dtype), laid_stride(forward_w(a), a.dtype)};
}

bool dz_is_dout(const fsdp_linear_grad_args& a) { return !a.times && a.activation == FSDP_ACT_NONE; }
Source grad_dz(const fsdp_linear_grad_args& a, bool kept, const void* at) {
    if (kept) return {at, a.m, a.n, lined(a.n, a.dtype), true};
    return {a.dout, a.m, a.n, row_stride(a.m, a.n, a.dout_stride), false};
}
// dx = dz weight, or dweight = dz^T x: `other` is weight or x.
Shape grad_shape(const fsdp_linear_grad_args& a, bool dweight, const Source& dz, const Source& other) {
    const int64_t first = laid_stride(dz, a.dtype), second = laid_stride(other, a.dtype);
    return dweight ? Shape{a.n, a.k, a.m, a.dtype, true, true, first, second}
                   : Shape{a.m, a.k, a.n, a.dtype, false, true, first, second};
}

// What a gradient needs besides its outputs.
struct GradParts {
    int64_t parts = 0, part_rows = 1;            // row parts of dbias
    int64_t dz = -1, dbias = -1;     // byte offsets
    int64_t bytes = 0;               // of the workspace
    Shape dx_shape, dw_shape;
    Source from_dz, weight, x;
    Cut dx, dw;
};

fsdp_status check_reach(const fsdp_linear_grad_args& a) {
    const Source dz = grad_dz(a, !dz_is_dout(a), nullptr);
    if (a.dx) {
        const fsdp_status st = check_reach(grad_shape(a, false, dz, {a.weight, a.n, a.k, row_stride(a.n, a.k, a.weight_stride), false}), linear_forms(a.dtype));
        if (st != FSDP_OK) return st;
    }
    return a.dweight ? check_reach(grad_shape(a, true, dz, {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false}), linear_forms(a.dtype)) : FSDP_OK;
}

GradParts parts_of(const fsdp_linear_grad_args& a, int cus, char* ws) {
    GradParts g;
    if (a.m > 0 && a.n > 0) {
        const int64_t columns = ceil_div(a.n, 512);
        g.part_rows = std::max<int64_t>(4, round_up(ceil_div(a.m * columns, 8 * int64_t(cus)), 4));
        g.parts = ceil_div(a.m, g.part_rows);
        if (!dz_is_dout(a) && (a.dx || a.dweight)) {
            g.dz = g.bytes;
            g.bytes += round_up(a.m * lined(a.n, a.dtype) * elem_bytes(a.dtype), 256);
        }
        if (a.dbias) {
            g.dbias = g.bytes;
            g.bytes += round_up(g.parts * a.n * 4, 256);
        }
    }
    g.from_dz = grad_dz(a, g.dz >= 0, ws + std::max<int64_t>(g.dz, 0));
    g.weight = {a.weight, a.n, a.k, row_stride(a.n, a.k, a.weight_stride), false};
    g.x = {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false};
    g.dx_shape = grad_shape(a, false, g.from_dz, g.weight);
    g.dw_shape = grad_shape(a, true, g.from_dz, g.x);
    const int64_t own = g.bytes;
    // The two products follow each other on the stream: they share what they need.
    if (a.dx) {
        g.dx = plan(g.dx_shape, g.from_dz, g.weight, cus, own);
        g.bytes = std::max(g.bytes, g.dx.bytes);
    }
    if (a.dweight) {
        g.dw = plan(g.dw_shape, g.from_dz, g.x, cus, own);
        g.bytes = std::max(g.bytes, g.dw.bytes);
    }
    return g;
}

}  // namespace
}  // namespace fsdp_block

using namespace fsdp_block;

extern "C" fsdp_status fsdp_block_linear_workspace(const fsdp_linear_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    fsdp_status st = check_linear(*args);
    if (st == FSDP_OK) st = check_reach(forward_shape(*args), linear_forms(args->dtype));
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    *bytes = plan(forward_shape(*args), forward_x(*args), forward_w(*args), cus, 0).bytes;
    return FSDP_OK;
}

extern "C" fsdp_status fsdp_block_linear(const fsdp_linear_args* args, void* workspace, int64_t workspace_bytes,
                                         hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_linear_args& a = *args;
    fsdp_status st = check_linear(a);
    if (st == FSDP_OK) st = check_reach(forward_shape(a), linear_forms(a.dtype));
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    const Shape s = forward_shape(a);
    const Source x = forward_x(a), w = forward_w(a);
    const Cut c = plan(s, x, w, cus, 0);
    if ((st = check_workspace(workspace, workspace_bytes, c.bytes)) != FSDP_OK) return st;
    const Epilogue e{a.bias, a.times, a.residual, a.pre, a.out, a.times_stride, a.residual_stride, a.pre_stride, a.out_stride,
                     a.activation};
    return run_product(s, x, w, e, c, static_cast<char*>(workspace), stream);
}

extern "C" fsdp_status fsdp_block_linear_grad_workspace(const fsdp_linear_grad_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    fsdp_status st = check_grad(*args);
    if (st == FSDP_OK) st = check_reach(*args);
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    *bytes = parts_of(*args, cus, nullptr).bytes;
    return FSDP_OK;
}

extern "C" fsdp_status fsdp_block_linear_grad(const fsdp_linear_grad_args* args, void* workspace, int64_t workspace_bytes,
                                              hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_linear_grad_args& a = *args;
    fsdp_status st = check_grad(a);
    if (st == FSDP_OK) st = check_reach(a);
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    char* const ws = static_cast<char*>(workspace);
    const GradParts g = parts_of(a, cus, ws);
    if ((st = check_workspace(workspace, workspace_bytes, g.bytes)) != FSDP_OK) return st;
    float* const part = g.dbias < 0 ? nullptr : reinterpret_cast<float*>(ws + g.dbias);
    if (a.m > 0 && a.n > 0 && (g.dz >= 0 || part || a.dtimes)) {
        const SlopeArgs s{a.dout, a.pre, a.times, g.dz >= 0 ? ws + g.dz : nullptr, a.dtimes, part, a.dout_stride,
                          a.pre_stride, a.times_stride, g.from_dz.stride, a.dtimes_stride, a.m, a.n, g.part_rows, a.activation};
        const dim3 grid(unsigned(ceil_div(a.n, 512)), unsigned(g.parts));
        st = with_type(a.dtype, [&](auto type) { return launch(slope_kernel<decltype(type)>, s, grid, 256, stream); });
        if (st != FSDP_OK) return st;
    }
    Join j(int(a.n));
    j.add(a.dbias, part, g.parts, a.dbias ? 1 : 0, a.dtype);
    if ((st = j.run(a.dtype, stream)) != FSDP_OK) return st;
    const auto plain = [](void* out, int64_t stride) {
        return Epilogue{nullptr, nullptr, nullptr, nullptr, out, 0, 0, 0, stride, FSDP_ACT_NONE};
    };
    if (a.dx) {
        st = run_product(g.dx_shape, g.from_dz, g.weight, plain(a.dx, a.dx_stride), g.dx, ws, stream);
        if (st != FSDP_OK) return st;
    }
    if (a.dweight) st = run_product(g.dw_shape, g.from_dz, g.x, plain(a.dweight, a.dweight_stride), g.dw, ws, stream);
    return st;
}
