// Matrices to 8 bits and back (include/fsdp_step.h).
//
// Bound by HBM: bf16 moves 3.03 bytes an element either way; 8192 x 4096 takes 22 us to
// save and 19 to restore, 4.6 and 5.4 TB/s.  A lane takes eight columns, so that four
// lanes hold a group and find its largest magnitude by two exchanges in the quad.

#include "step_saved.h"

#include <algorithm>

namespace fsdp_block {
namespace {

// A lane takes eight columns, a quad a group of 32. Items of a wave are 64 times eight columns,
// kTogether neighbouring ones, all asked for before the first is worked on: a run of 512 columns of
// a row, `runs` to a row; or (runs is 0) whole groups of one row after the other, `per` times
// eight columns to a row: of rows of less than 512 columns, whose runs would leave lanes idle.
constexpr int kTogether = 4;
struct Places {
    int64_t rows, cols, runs, per, items;
};
Places places(int64_t rows, int64_t cols) {
    const int64_t per = ceil_div(cols, FSDP_STEP_GROUP) * 4;
    return per < 64 ? Places{rows, cols, 0, per, ceil_div(rows * per, 64)} : Places{rows, cols, ceil_div(cols, 512), 0, rows * ceil_div(cols, 512)};
}
struct Place {
    int64_t row, j;
    int left;                        // columns from j on; 0 and less: none
};
template <typename F>
__device__ __forceinline__ void for_items(const Places& p, F f) {
    for (int64_t first = (int64_t(blockIdx.x) * 4 + threadIdx.x / 64) * kTogether; first < p.items; first += int64_t(gridDim.x) * 4 * kTogether) {
        Place at[kTogether];
        if (p.runs) {
            int64_t row = first / p.runs, run = first - row * p.runs;
#pragma unroll
            for (int u = 0; u < kTogether; ++u) {
                at[u] = {row, (run * 64 + threadIdx.x % 64) * 8, 0};
                at[u].left = first + u < p.items ? int(min(p.cols - at[u].j, int64_t(8))) : -1;
                if (++run == p.runs) {
                    run = 0;
                    ++row;
                }
            }
        } else {
            const int64_t row0 = first * 64 / p.per;
            const uint32_t unit0 = uint32_t(first * 64 - row0 * p.per) + threadIdx.x % 64, per = uint32_t(p.per);
#pragma unroll
            for (int u = 0; u < kTogether; ++u) {
                const uint32_t down = (unit0 + 64 * u) / per;
                at[u] = {row0 + down, int64_t(unit0 + 64 * u - down * per) * 8, 0};
                at[u].left = at[u].row < p.rows ? int(min(p.cols - at[u].j, int64_t(8))) : -1;
            }
        }
        f(at);
    }
}

struct SaveArgs {
    const void* x;
    int8_t* codes;
    uint8_t* scales;
    int64_t x_stride, codes_stride, scales_stride;
    Places places;
};

template <typename T>
__global__ __launch_bounds__(256) void save_kernel(const SaveArgs a) {
    for_items(a.places, [&](const Place (&at)[kTogether]) {
        Eight<T> in[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const T* const x = static_cast<const T*>(a.x) + at[u].row * a.x_stride + at[u].j;
            if (at[u].left >= 8) in[u] = load8_once(x);
            else in[u] = load_some(x, at[u].left);
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = float(in[u][c]);
            save8(v, at[u].left, a.codes + at[u].row * a.codes_stride + at[u].j,
                  a.scales + at[u].row * a.scales_stride + at[u].j / FSDP_STEP_GROUP);
        }
    });
}

struct RestoreArgs {
    const int8_t* codes;
    const uint8_t* scales;
    void* x;
    int64_t codes_stride, scales_stride, x_stride, cols;
    Places places;                   // of x, with its zeros after `cols`
};

// Columns cols .. to_cols - 1 become zeros.
template <typename T>
__global__ __launch_bounds__(256) void restore_kernel(const RestoreArgs a) {
    for_items(a.places, [&](const Place (&at)[kTogether]) {
        i8x8 q[kTogether];
        float scale[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int left = at[u].left > 0 ? int(min(a.cols - at[u].j, int64_t(8))) : 0;
            const int8_t* const codes = a.codes + at[u].row * a.codes_stride + at[u].j;
            if (left >= 8) q[u] = load_codes_once(codes);
            else q[u] = load_codes(codes, left);
            scale[u] = left > 0 ? scale_value(a.scales[at[u].row * a.scales_stride + at[u].j / FSDP_STEP_GROUP]) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = at[u].j + c < a.cols ? float(q[u][c]) * scale[u] : 0.f;
            if (at[u].left > 0) store_some(static_cast<T*>(a.x) + at[u].row * a.x_stride + at[u].j, at[u].left, v);
        }
    });
}

fsdp_status check(int64_t rows, int64_t cols, fsdp_dtype dtype) {
    if (rows < 0 || cols < 0) return fail(FSDP_ERR_INVALID, "rows and cols must not be negative");
    if (!known_dtype(dtype)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (rows > INT32_MAX || cols > 1 << 30) return fail(FSDP_ERR_OVERFLOW, "rows is above 2^31 or cols above 2^30");
    return FSDP_OK;
}

template <typename F>
fsdp_status with_type(fsdp_dtype dtype, F f) {
    return dtype == FSDP_DTYPE_BF16 ? f(bf16(0.f)) : dtype == FSDP_DTYPE_F16 ? f(f16(0.f)) : f(0.f);
}

}  // namespace

fsdp_status restore(const void* codes, int64_t codes_stride, const void* scales, int64_t scales_stride, void* x, int64_t x_stride,
                    int64_t rows, int64_t cols, int64_t to_cols, fsdp_dtype dtype, hipStream_t stream) {
    if (rows == 0 || to_cols == 0) return FSDP_OK;
    const Places p = places(rows, to_cols);
    const RestoreArgs k{static_cast<const int8_t*>(codes), static_cast<const uint8_t*>(scales), x, codes_stride, scales_stride,
                        x_stride, cols, p};
    const dim3 grid(unsigned(std::min<int64_t>(ceil_div(p.items, 4 * kTogether), 1 << 16)));
    return with_type(dtype, [&](auto type) { return launch(restore_kernel<decltype(type)>, k, grid, 256, stream); });
}

}  // namespace fsdp_block

using namespace fsdp_block;

extern "C" fsdp_status fsdp_step_save(const fsdp_step_save_args* args, hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_step_save_args& a = *args;
    fsdp_status st = check(a.rows, a.cols, a.dtype);
    if (st != FSDP_OK) return st;
    Checked c;
    c.add("x", a.x, a.rows, a.cols, a.x_stride, a.dtype, true);
    c.add("codes", a.codes, a.rows, a.cols, a.codes_stride, kBytes, true, true);
    c.add("scales", a.scales, a.rows, ceil_div(a.cols, FSDP_STEP_GROUP), a.scales_stride, kBytes, true, true);
    if ((st = c.done()) != FSDP_OK || a.rows == 0 || a.cols == 0) return st;
    const Places p = places(a.rows, a.cols);
    const SaveArgs k{a.x, static_cast<int8_t*>(a.codes), static_cast<uint8_t*>(a.scales), a.x_stride, a.codes_stride,
                     a.scales_stride, p};
    const dim3 grid(unsigned(std::min<int64_t>(ceil_div(p.items, 4 * kTogether), 1 << 16)));
    return with_type(a.dtype, [&](auto type) { return launch(save_kernel<decltype(type)>, k, grid, 256, stream); });
}

extern "C" fsdp_status fsdp_step_restore(const fsdp_step_restore_args* args, hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_step_restore_args& a = *args;
    fsdp_status st = check(a.rows, a.cols, a.dtype);
    if (st != FSDP_OK) return st;
    Checked c;
    c.add("codes", a.codes, a.rows, a.cols, a.codes_stride, kBytes, true);
    c.add("scales", a.scales, a.rows, ceil_div(a.cols, FSDP_STEP_GROUP), a.scales_stride, kBytes, true);
    c.add("x", a.x, a.rows, a.cols, a.x_stride, a.dtype, true, true);
    if ((st = c.done()) != FSDP_OK || a.rows == 0 || a.cols == 0) return st;
    return restore(a.codes, a.codes_stride, a.scales, a.scales_stride, a.x, a.x_stride, a.rows, a.cols, a.cols, a.dtype, stream);
}
