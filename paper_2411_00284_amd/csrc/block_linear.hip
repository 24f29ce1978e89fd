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

#include "block_product.h"
#include "block_join.h"

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

// ------------------------------------------------------------------ onto the grid

// Copies matrices to rows of whole lines, zeros after their columns up to a whole
// 16-byte unit.  Sizes in halves of 32 bits, which fp32 elements are two of.  A
// wave takes 64 units of a row, so that the division is one for all of them.
struct PadArgs {
    const uint16_t* from[2];
    uint16_t* to[2];
    int64_t rows[2], cols[2], stride[2], to_stride[2];
    uint32_t runs[2];                // of 64 units, in a row
};

__global__ __launch_bounds__(256) void pad_kernel(const PadArgs a) {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(2))) any {
        u16x8 v;
    };
    const uint32_t first = uint32_t(a.rows[0]) * a.runs[0], all = first + uint32_t(a.rows[1]) * a.runs[1];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
    for (uint32_t item = wave; item < all; item += gridDim.x * 4) {
        const int which = item >= first;
        const uint32_t run = which ? item - first : item, row = run / a.runs[which];
        const int64_t j = (int64_t(run - row * a.runs[which]) * 64 + threadIdx.x % 64) * 8, left = a.cols[which] - j;
        if (left <= 0) continue;
        const uint16_t* at = a.from[which] + row * a.stride[which] + j;
        u16x8 v;
        if (left >= 8) {
            v = reinterpret_cast<const any*>(at)->v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < left ? at[e] : uint16_t(0);
        }
        *reinterpret_cast<u16x8*>(a.to[which] + row * a.to_stride[which] + j) = v;
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

template <typename F>
fsdp_status with_type(fsdp_dtype dtype, F f) {
    return dtype == FSDP_DTYPE_BF16 ? f(bf16(0.f)) : dtype == FSDP_DTYPE_F16 ? f(f16(0.f)) : f(0.f);
}

// The forms of a product in tiles.  Times in us of a step (64 k, fp32: 32) on one
// MI355X: `alone` with one workgroup on a CU, `full` with `held` of them on every
// CU, and `fixed` for the start and the end of a tile, as measured over products from
// 16 x 14336 x 4096 to 8192 x 28672 x 8192.  A guide, not a prediction: 64 x 64 tiles
// of 771 x 1153 x 2501 take 0.4 us a step.  Those of fp32 are from 2048 x 1024 x 688 and
// 4096^3 only: dx of the former is expected at 24 us and takes 33.
struct Form {
    int tile_m, tile_n, steps, held;
    double alone, full, fixed;
};
constexpr Form kForms16[] = {
    {256, 256, 2, 1, 1.15, 1.60, 6.0},
    {128, 128, 2, 2, 0.60, 0.97, 4.0},
    {128, 128, 4, 1, 0.36, 0.52, 3.5},
    {64, 128, 4, 1, 0.25, 0.32, 3.5},
    {64, 64, 8, 1, 0.14, 0.20, 3.5},
};
constexpr Form kForms32[] = {
    {128, 128, 2, 2, 1.80, 3.60, 4.0},
    {64, 128, 4, 1, 0.95, 0.95, 3.5},
};

// How one product is run.
struct Cut {
    const Form* form = nullptr;      // NULL: row_kernel
    int count = 1;                   // parts of k
    int64_t part_k = 0;
    // Not NULL: the rows (columns) of out from rest_at on are a launch of their own.
    const Form* rest = nullptr;
    bool rest_rows = false;
    int64_t rest_at = 0;
    // Byte offsets in the workspace and its size: the operands laid on the grid, the parts.
    int64_t pad_a = -1, pad_b = -1, parts = -1, bytes = 0;
};

struct Shape {
    int64_t m, n, k;
    fsdp_dtype dtype;
    bool columns_a, columns_b;
    int64_t stride_a, stride_b;      // of the operands as they are laid on the grid
};

// The most bytes that a load may lie from its tile's first (Operand::load), and
// whether a form's loads stay within: an operand by rows has the tile's rows in a
// step, one by columns the step's rows of k.
constexpr int64_t kReach = 0x7ffffff0;
bool reaches(const Form& f, const Shape& s) {
    const int64_t size = elem_bytes(s.dtype), deep = 128 / size;
    const auto end = [&](bool columns, int64_t rows, int64_t tile, int64_t stride) {
        return columns ? ((std::min(deep, s.k) - 1) * stride + tile) * size : (std::min(tile, rows) - 1) * stride * size + 128;
    };
    return end(s.columns_a, s.m, f.tile_m, s.stride_a) <= kReach && end(s.columns_b, s.n, f.tile_n, s.stride_b) <= kReach;
}

constexpr int64_t kMostRows = 4;     // of row_kernel
// Below 2^27 columns: eight or sixteen of them to a workgroup must make fewer than 2^32 threads.
bool row_form(const Shape& s) { return s.m <= kMostRows && s.n < (int64_t(1) << 27) && !s.columns_a && !s.columns_b; }

// Bytes per us in which the operands come out of memory, in all and to one
// workgroup, and what the caches keep of them: with the second bound, which wants
// 220 workgroups, 64 x 14336 -> 4096 takes 29.5 us instead of 45, 64 x 28672 -> 8192
// 104 instead of 140; under 16 MB it would cut products for nothing (64 x 1024 -> 1024
// 9.1 us instead of 7.2).
constexpr double kMostRead = 5.5e6, kGroupRead = 0.025e6, kCached = 16e6;

// Of whole rounds of workgroups and the last one.
double rounds_time(const Form& form, int64_t groups, int64_t steps, int cus) {
    const int64_t slots = int64_t(cus) * form.held, whole = groups / slots, rest = groups - whole * slots;
    const double time = double(whole) * (double(steps) * form.full + form.fixed);
    return rest ? time + double(steps) * (rest > cus ? form.full : form.alone) + form.fixed : time;
}

// The form and the cut with the least expected time: whole rounds of workgroups
// over the CUs, the fullest CU of the last round, reading the operands if that takes
// longer, and the join of the parts (3 us, and 8 bytes moved per value and part).
// Up to four rows of x, row_kernel reads the weight at HBM's rate in one launch.
// Tiles of 256 x 256 that leave a last round of few are cut where the whole rounds
// end, and the rest of out takes tiles of 128 x 128 in a second launch (3 us): bf16
// 6144 x 6144 x 4096 takes 281 us instead of 301, 14336 x 4096 with k = 8192 746
// instead of 791.  (Smaller tiles for the rest: 334 instead of 300 us at 5000^3.)
Cut choose(const Shape& s, int cus) {
    Cut best;
    if (row_form(s)) return best;
    const bool wide = s.dtype == FSDP_DTYPE_F32;
    const Form* const forms = wide ? kForms32 : kForms16;
    const int step_k = wide ? 32 : 64;
    const int64_t steps = std::max<int64_t>(1, ceil_div(s.k, step_k));
    const double read = double(elem_bytes(s.dtype)) * (double(s.m) * double(s.k) + double(s.n) * double(s.k));
    const double joining = double(s.m) * double(s.n) * 8 / 5e6;
    double least = 0;
    for (int f = 0; f < (wide ? 2 : 5); ++f) {
        const Form& form = forms[f];
        if (!reaches(form, s)) continue;
        const int64_t tiles = ceil_div(s.m, form.tile_m) * ceil_div(s.n, form.tile_n);
        for (int parts = 1; parts <= 16; ++parts) {
            // Parts of at least four steps, and no more of them than some rounds.
            if (parts > 1 && (steps < 4 * parts || tiles * (parts - 1) > 3 * int64_t(cus))) break;
            const int64_t each = (steps + parts - 1) / parts, count = (steps + each - 1) / each;
            if (count != parts) continue;
            const int64_t groups = tiles * parts;
            double time = rounds_time(form, groups, each, cus);
            const double rate = read > kCached ? std::min(kMostRead, kGroupRead * double(groups)) : kMostRead;
            time = std::max(time, read / rate + form.fixed);
            if (parts > 1) time += 3.0 + double(parts) * joining;
            if (!best.form || time < least) {
                least = time;
                best.form = &form;
                best.part_k = each * step_k;
                best.count = parts;
            }
        }
    }
    if (wide || s.m == 0 || s.n == 0) return best;
    const Form &big = forms[0], &small = forms[1];
    if (!reaches(big, s)) return best;
    const int64_t down = ceil_div(s.m, big.tile_m), across = ceil_div(s.n, big.tile_n);
    for (const bool rows : {true, false}) {
        // Rows (columns) of tiles in whole rounds, and what is left of out.
        const int64_t other = rows ? across : down, taken = down * across / cus * cus / other;
        const int64_t at = taken * (rows ? big.tile_m : big.tile_n), m = rows ? s.m - at : s.m, n = rows ? s.n : s.n - at;
        if (taken == 0 || m <= 0 || n <= 0) continue;
        const double time = rounds_time(big, taken * other, steps, cus) + 3.0 +
                            rounds_time(small, ceil_div(m, small.tile_m) * ceil_div(n, small.tile_n), steps, cus);
        if (time >= least) continue;
        least = time;
        best = Cut{};
        best.form = &big;
        best.part_k = steps * step_k;
        best.rest = &small;
        best.rest_rows = rows;
        best.rest_at = at;
    }
    return best;
}

struct Source {
    const void* p;
    int64_t rows, cols, stride;      // as it lies in memory
    bool zeros;                      // zeros follow a row, up to a whole 16-byte unit
};

// Elements of a row laid out in whole lines.
int64_t lined(int64_t cols, fsdp_dtype dtype) { return round_up(cols, 128 / elem_bytes(dtype)); }

// Whether an operand lies on the 16-byte grid in whole units, as product_kernel
// reads it, with the offsets of a step in 31 bits.
bool on_grid(const Source& o, fsdp_dtype dtype) {
    const int unit = 16 / elem_bytes(dtype);
    return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && o.stride % unit == 0 && o.stride < (1 << 21) && (o.zeros || o.cols % unit == 0);
}

// A row's stride where product_kernel reads it.
int64_t laid_stride(const Source& o, fsdp_dtype dtype) { return on_grid(o, dtype) ? o.stride : lined(o.cols, dtype); }

// Whether any form reaches the operands (row_kernel reaches all of its).
fsdp_status check_reach(const Shape& s) {
    if (s.m == 0 || s.n == 0 || row_form(s)) return FSDP_OK;
    if (s.dtype == FSDP_DTYPE_F32 ? reaches(kForms32[1], s) : reaches(kForms16[4], s)) return FSDP_OK;
    return fail(FSDP_ERR_OVERFLOW, "a tile's rows of an operand of %lld x %lld, %lld x %lld do not lie within 2^31 bytes",
                (long long)s.m, (long long)s.k, (long long)s.n, (long long)s.k);
}

// Adds a product's needs to those of `bytes`.
Cut plan(const Shape& s, const Source& a, const Source& b, int cus, int64_t bytes) {
    Cut c = choose(s, cus);
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
    if (c.pad_a >= 0 || c.pad_b >= 0) {
        PadArgs pad{};
        const int halves = elem_bytes(s.dtype) / 2;
        const auto lay = [&](int which, const Source& o, int64_t at, const void** to, int64_t* stride) {
            pad.runs[which] = 1;
            if (at < 0) return;
            pad.from[which] = static_cast<const uint16_t*>(o.p);
            pad.to[which] = reinterpret_cast<uint16_t*>(ws + at);
            pad.rows[which] = o.rows;
            pad.cols[which] = o.cols * halves;
            pad.stride[which] = o.stride * halves;
            pad.to_stride[which] = lined(o.cols, s.dtype) * halves;
            pad.runs[which] = uint32_t(ceil_div(pad.cols[which], 512));
            *to = ws + at;
            *stride = lined(o.cols, s.dtype);
        };
        lay(0, a, c.pad_a, &p.a, &p.a_stride);
        lay(1, b, c.pad_b, &p.b, &p.b_stride);
        const int64_t runs = pad.rows[0] * pad.runs[0] + pad.rows[1] * pad.runs[1];
        // check_sizes bounds rows x cols by 2^34 and rows by 2^28: the runs fit 31 bits.
        if ((st = launch(pad_kernel, pad, dim3(unsigned(std::min<int64_t>(ceil_div(runs, 4), 1 << 16))), 256, stream)) != FSDP_OK)
            return st;
    }
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
    if (m > INT32_MAX / 2 || n > INT32_MAX / 2 || k > INT32_MAX / 2) return fail(FSDP_ERR_OVERFLOW, "a size is above 2^30");
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
        const fsdp_status st = check_reach(grad_shape(a, false, dz, {a.weight, a.n, a.k, row_stride(a.n, a.k, a.weight_stride), false}));
        if (st != FSDP_OK) return st;
    }
    return a.dweight ? check_reach(grad_shape(a, true, dz, {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false})) : FSDP_OK;
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
    if (st == FSDP_OK) st = check_reach(forward_shape(*args));
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
    if (st == FSDP_OK) st = check_reach(forward_shape(a));
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
