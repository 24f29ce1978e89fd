// Host side shared by the block operators: the error text, argument checks and
// the launch helper.  Nothing here allocates or throws: the entry points are
// called from C.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "fsdp_block.h"

namespace fsdp_block {

// Sets this thread's error text (printf style) and returns `st`.
fsdp_status fail(fsdp_status st, const char* format, ...) __attribute__((format(printf, 2, 3)));
// Forgets the error text: every entry point begins with it.
void clear_error();
// Compute units of the current device; 0 with *st set when HIP cannot say.
int cu_count(fsdp_status* st);

inline bool known_dtype(fsdp_dtype t) { return t == FSDP_DTYPE_BF16 || t == FSDP_DTYPE_F32 || t == FSDP_DTYPE_F16; }
inline int elem_bytes(fsdp_dtype t) { return t == FSDP_DTYPE_F32 ? 4 : 2; }

// One matrix argument of a call.
struct Matrix {
    const char* name;
    const void* p;
    int64_t rows, cols, stride;      // stride in elements; rows of `cols` contiguous elements
    fsdp_dtype dtype;
    int esize;
    bool output;
    bool in_place;                   // an input that a kernel reads where it writes, and nowhere else
    const void* alias[2];            // inputs that this output may be
    int64_t lo() const { return int64_t(reinterpret_cast<uintptr_t>(p)); }
    bool empty() const { return rows == 0 || cols == 0; }
    int64_t bytes() const { return ((rows - 1) * stride + cols) * esize; }   // from its first to past its last element
};

// The matrices of one call, checked as they are added and against each other
// at the end.
class Checked {
public:
    // `needed`: may not be NULL unless it is empty.  A NULL matrix is left out.
    // An output takes the inputs it may be, which must have its stride and type.
    void add(const char* name, const void* p, int64_t rows, int64_t cols, int64_t stride, fsdp_dtype dtype, bool needed,
             bool output = false, const void* alias0 = nullptr, const void* alias1 = nullptr);
    // An input that an output may be: every value is read before it is written, by the
    // thread or workgroup that writes it.  Others may not lie there, whatever their address
    // (a gate's row that is the first row of the stream, x that is the residual too).
    void add_in_place(const char* name, const void* p, int64_t rows, int64_t cols, int64_t stride, fsdp_dtype dtype, bool needed) {
        const int before = n_;
        add(name, p, rows, cols, stride, dtype, needed);
        if (n_ > before) m_[before].in_place = true;
    }
    void add_vector(const char* name, const void* p, int64_t n, fsdp_dtype dtype, bool needed, bool output = false) {
        add(name, p, n > 0 ? 1 : 0, n, n, dtype, needed, output);
    }
    // The first error found, or FSDP_OK; checks for overlap.
    fsdp_status done();

private:
    static constexpr int kMost = 16;
    Matrix m_[kMost];
    int n_ = 0;
    fsdp_status st_ = FSDP_OK;
};

// One launch; `grid` is cut to what a launch may hold, kernels loop beyond it
// where they say so.
template <typename Args>
fsdp_status launch(void (*kernel)(const Args), const Args& args, dim3 grid, int block, hipStream_t stream, unsigned lds = 0) {
    void* kargs[] = {const_cast<Args*>(&args)};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), kargs, lds, stream);
    if (e != hipSuccess) return fail(FSDP_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
    return FSDP_OK;
}

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

fsdp_status check_workspace(const void* workspace, int64_t held, int64_t needed);

}  // namespace fsdp_block
