// Matrices to 8 bits and back (include/fsdp_step.h).
//
// Bound by HBM: bf16 moves 3.03 bytes an element either way.  A lane takes eight
// columns, so that four lanes hold a group and find its largest magnitude by two
// exchanges in the quad; a wave takes a run of 512 columns of a row.

#include "step_saved.h"

#include <algorithm>

namespace fsdp_block {
namespace {

struct SaveArgs {
    const void* x;
    int8_t* codes;
    uint8_t* scales;
    int64_t x_stride, codes_stride, scales_stride, cols, runs, items;
};

template <typename T>
__global__ __launch_bounds__(256) void save_kernel(const SaveArgs a) {
    for (int64_t item = int64_t(blockIdx.x) * 4 + threadIdx.x / 64; item < a.items; item += int64_t(gridDim.x) * 4) {
        const int64_t row = item / a.runs, j = ((item - row * a.runs) * 64 + threadIdx.x % 64) * 8;
        const int left = int(min(a.cols - j, int64_t(8)));
        float v[8] = {};
        if (left > 0) {
            const Eight<T> in = load_some(static_cast<const T*>(a.x) + row * a.x_stride + j, left);
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = float(in[c]);
        }
        save8(v, left, a.codes + row * a.codes_stride + j, a.scales + row * a.scales_stride + j / FSDP_STEP_GROUP);
    }
}

struct RestoreArgs {
    const int8_t* codes;
    const uint8_t* scales;
    void* x;
    int64_t codes_stride, scales_stride, x_stride, cols, to_cols, runs, items;
};

// Columns cols .. to_cols - 1 become zeros.
template <typename T>
__global__ __launch_bounds__(256) void restore_kernel(const RestoreArgs a) {
    for (int64_t item = int64_t(blockIdx.x) * 4 + threadIdx.x / 64; item < a.items; item += int64_t(gridDim.x) * 4) {
        const int64_t row = item / a.runs, j = ((item - row * a.runs) * 64 + threadIdx.x % 64) * 8;
        const int left = int(min(a.cols - j, int64_t(8))), write = int(min(a.to_cols - j, int64_t(8)));
        if (write <= 0) continue;
        float v[8] = {};
        if (left > 0) {
            const i8x8 q = load_codes(a.codes + row * a.codes_stride + j, left);
            const float scale = scale_value(a.scales[row * a.scales_stride + j / FSDP_STEP_GROUP]);
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = c < left ? float(q[c]) * scale : 0.f;
        }
        store_some(static_cast<T*>(a.x) + row * a.x_stride + j, write, v);
    }
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
    const int64_t runs = ceil_div(to_cols, 512), items = rows * runs;
    if (items == 0) return FSDP_OK;
    const RestoreArgs k{static_cast<const int8_t*>(codes), static_cast<const uint8_t*>(scales), x, codes_stride, scales_stride,
                        x_stride, cols, to_cols, runs, items};
    const dim3 grid(unsigned(std::min<int64_t>(ceil_div(items, 4), 1 << 16)));
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
    const int64_t runs = ceil_div(a.cols, 512), items = a.rows * runs;
    const SaveArgs k{a.x, static_cast<int8_t*>(a.codes), static_cast<uint8_t*>(a.scales), a.x_stride, a.codes_stride,
                     a.scales_stride, a.cols, runs, items};
    const dim3 grid(unsigned(std::min<int64_t>(ceil_div(items, 4), 1 << 16)));
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
