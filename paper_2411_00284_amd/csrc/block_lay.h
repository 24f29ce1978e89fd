// Lays matrices on the 16-byte grid, for the matrix products.
#pragma once

#include "block_cut.h"

namespace fsdp_block {
namespace {

// Copies matrices to rows of whole lines, zeros after their columns up to a whole
// 16-byte unit.  Sizes in halves of 32 bits, which fp32 elements are two of.  A
// wave takes 64 units of a row, so that the division is one for all of them.
template <int kMost>
struct PadArgs {
    const uint16_t* from[kMost];
    uint16_t* to[kMost];
    int64_t rows[kMost], cols[kMost], stride[kMost], to_stride[kMost];
    uint32_t runs[kMost];                // of 64 units, in a row
};

template <int kMost>
__global__ __launch_bounds__(256) void pad_kernel(const PadArgs<kMost> a) {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    struct __attribute__((packed, aligned(2))) any {
        u16x8 v;
    };
    uint32_t first[kMost + 1] = {};              // each matrix's first run
#pragma unroll
    for (int w = 0; w < kMost; ++w) first[w + 1] = first[w] + uint32_t(a.rows[w]) * a.runs[w];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
    for (uint32_t item = wave; item < first[kMost]; item += gridDim.x * 4) {
        int which = 0;
#pragma unroll
        for (int w = 1; w < kMost; ++w) which += item >= first[w];
        const uint32_t run = item - first[which], row = run / a.runs[which];
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

// The copies of one launch, of up to kMost matrices.
template <int kMost>
class Pads {
public:
    Pads() {
        for (int w = 0; w < kMost; ++w) a_.runs[w] = 1;
    }
    // `o` to rows of whole lines at `to`.
    void add(const Source& o, fsdp_dtype dtype, char* to) {
        const int halves = elem_bytes(dtype) / 2;
        a_.from[n_] = static_cast<const uint16_t*>(o.p);
        a_.to[n_] = reinterpret_cast<uint16_t*>(to);
        a_.rows[n_] = o.rows;
        a_.cols[n_] = o.cols * halves;
        a_.stride[n_] = o.stride * halves;
        a_.to_stride[n_] = lined(o.cols, dtype) * halves;
        a_.runs[n_] = uint32_t(ceil_div(a_.cols[n_], 512));
        runs_ += o.rows * a_.runs[n_++];
    }
    // The runs have to fit 31 bits: the products bound rows x cols by 2^34 and rows by 2^28.
    fsdp_status run(hipStream_t stream) const {
        if (runs_ == 0) return FSDP_OK;
        return launch(pad_kernel<kMost>, a_, dim3(unsigned(std::min<int64_t>(ceil_div(runs_, 4), 1 << 16))), 256, stream);
    }

private:
    PadArgs<kMost> a_{};
    int n_ = 0;
    int64_t runs_ = 0;
};

}  // namespace
}  // namespace fsdp_block
