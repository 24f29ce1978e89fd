// Joins column sums that workgroups made over parts of the rows (fp32, one row
// of the workspace each) into gradients, in the order of the parts.
#pragma once

#include "block_device.h"
#include "block_host.h"

#include <algorithm>

namespace fsdp_block {
namespace {

struct JoinArgs {
    const float* part[3];
    void* out[3];
    int64_t units[3];                            // rows of `part` that make one output row
    int rows[3];                                 // output rows; blockIdx.y counts those of all outputs
    int f32[3];
    int hidden;
};

// A line of 32 columns per workgroup and 32 rows of parts at a time: many
// workgroups, each with few loads to wait for one after the other.
constexpr int kJoinColumns = 32, kJoinThreads = 1024;
constexpr int64_t kJoinGrid = int64_t(1) << 21;      // workgroups along the columns: below 2^32 threads

template <typename TB>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const JoinArgs a) {
    constexpr int kParts = kJoinThreads / kJoinColumns;
    __shared__ float sums[kParts][kJoinColumns];
    int row = blockIdx.y, which = 0;
    while (row >= a.rows[which]) row -= a.rows[which++];
    const int p = threadIdx.x / kJoinColumns;
    const int64_t units = a.units[which];
    const float* const part = a.part[which] + int64_t(row) * units * a.hidden;
    for (int first = blockIdx.x * kJoinColumns; first < a.hidden; first += gridDim.x * kJoinColumns) {
        const int column = first + threadIdx.x % kJoinColumns;
        float s = 0.f;
        if (column < a.hidden)
#pragma unroll 8
            for (int64_t u = p; u < units; u += kParts) s += part[u * a.hidden + column];
        sums[p][threadIdx.x % kJoinColumns] = s;
        __syncthreads();
        if (p == 0 && column < a.hidden) {
            s = 0.f;
#pragma unroll
            for (int k = 0; k < kParts; ++k) s += sums[k][threadIdx.x];
            if (a.f32[which]) static_cast<float*>(a.out[which])[int64_t(row) * a.hidden + column] = s;
            else static_cast<TB*>(a.out[which])[int64_t(row) * a.hidden + column] = TB(s);
        }
        __syncthreads();                             // the sums are the next columns'
    }
}

// Up to three outputs of one launch.
class Join {
public:
    explicit Join(int hidden) { a_.hidden = hidden; }
    // `out` [rows, hidden] (or NULL) = sums of `units` rows of `part` each.
    void add(void* out, const float* part, int64_t units, int64_t rows, fsdp_dtype dtype) {
        if (!out || rows == 0) return;
        a_.part[n_] = part;
        a_.out[n_] = out;
        a_.units[n_] = units;
        a_.rows[n_] = int(rows);
        a_.f32[n_++] = dtype == FSDP_DTYPE_F32;
        rows_ += rows;
    }
    // `dtype`: that of the outputs that are not fp32.
    fsdp_status run(fsdp_dtype dtype, hipStream_t stream) const {
        if (n_ == 0 || a_.hidden == 0) return FSDP_OK;
        const dim3 grid(unsigned(std::min(ceil_div(a_.hidden, kJoinColumns), kJoinGrid)), unsigned(rows_));
        return dtype == FSDP_DTYPE_BF16 ? launch(join_kernel<bf16>, a_, grid, kJoinThreads, stream)
               : dtype == FSDP_DTYPE_F16 ? launch(join_kernel<f16>, a_, grid, kJoinThreads, stream)
                                         : launch(join_kernel<float>, a_, grid, kJoinThreads, stream);
    }

private:
    JoinArgs a_{};
    int n_ = 0;
    int64_t rows_ = 0;
};

}  // namespace
}  // namespace fsdp_block
