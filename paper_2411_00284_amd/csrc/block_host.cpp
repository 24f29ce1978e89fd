// Argument checks and error text of the block operators (host code).

#include "block_host.h"

#include <atomic>
#include <cstdarg>
#include <cstdio>

namespace fsdp_block {
namespace {

constexpr int64_t kMaxBytes = int64_t(1) << 62;
thread_local char t_text[256] = "";

// Whether two matrices share a byte.  Matrices of one row stride may interleave
// (column slices of one buffer); of two strides, their whole spans count.
bool overlap(const Matrix& a, const Matrix& b) {
    if (a.empty() || b.empty()) return false;
    if (a.lo() + a.bytes() <= b.lo() || b.lo() + b.bytes() <= a.lo()) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    const int64_t step = a.rows > 1 ? a.stride * a.esize : b.stride * b.esize;
    if ((a.rows > 1 && b.rows > 1 && a.stride * a.esize != b.stride * b.esize) || step == 0) return true;
    const int64_t d = ((b.lo() - a.lo()) % step + step) % step;      // b's rows start d bytes after a's
    return d < a.cols * a.esize || d + b.cols * b.esize > step;
}

}  // namespace

fsdp_status fail(fsdp_status st, const char* format, ...) {
    va_list args;
    va_start(args, format);
    vsnprintf(t_text, sizeof t_text, format, args);
    va_end(args);
    return st;
}

void clear_error() { t_text[0] = 0; }

int cu_count(fsdp_status* st) {
    static std::atomic<int> cache[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) {
        *st = fail(FSDP_ERR_HIP, "hipGetDevice failed");
        return 0;
    }
    if (dev >= 0 && dev < 64) {
        const int c = cache[dev].load(std::memory_order_relaxed);
        if (c > 0) return c;
    }
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
        *st = fail(FSDP_ERR_HIP, "hipDeviceGetAttribute(multiProcessorCount) failed");
        return 0;
    }
    if (dev >= 0 && dev < 64) cache[dev].store(n, std::memory_order_relaxed);
    return n;
}

void Checked::add(const char* name, const void* p, int64_t rows, int64_t cols, int64_t stride, fsdp_dtype dtype, bool needed,
                  bool output, const void* alias0, const void* alias1) {
    if (st_ != FSDP_OK) return;
    const int esize = elem_bytes(dtype);
    const bool empty = rows == 0 || cols == 0;
    if (!p) {
        if (needed && !empty) st_ = fail(FSDP_ERR_INVALID, "%s is NULL", name);
        return;
    }
    if (reinterpret_cast<uintptr_t>(p) % uintptr_t(esize) != 0) {
        st_ = fail(FSDP_ERR_ALIGN, "%s is not element-aligned", name);
        return;
    }
    if (rows <= 1) stride = cols;
    if (rows > 1 && stride < cols) {
        st_ = fail(FSDP_ERR_INVALID, "%s: rows of %lld elements at a stride of %lld", name, (long long)cols, (long long)stride);
        return;
    }
    int64_t span = 0;
    if (!empty && (__builtin_mul_overflow(rows, stride, &span) || span > kMaxBytes / esize)) {
        st_ = fail(FSDP_ERR_OVERFLOW, "%s: its size does not fit", name);
        return;
    }
    if (n_ == kMost) {
        st_ = fail(FSDP_ERR_TOO_MANY, "too many arguments to check");
        return;
    }
    m_[n_++] = {name, p, rows, cols, stride, dtype, esize, output, false, {alias0, alias1}};
}

fsdp_status Checked::done() {
    for (int i = 0; i < n_ && st_ == FSDP_OK; ++i) {
        if (!m_[i].output) continue;
        for (int j = 0; j < n_; ++j) {
            if (j == i || (m_[j].output && j < i) || !overlap(m_[i], m_[j])) continue;
            const bool same = m_[i].p == m_[j].p && m_[i].stride == m_[j].stride && m_[i].dtype == m_[j].dtype;
            if (m_[j].in_place && same && (m_[i].alias[0] == m_[j].p || m_[i].alias[1] == m_[j].p)) continue;
            st_ = fail(FSDP_ERR_OVERLAP, "%s overlaps %s", m_[i].name, m_[j].name);
            break;
        }
    }
    return st_;
}

fsdp_status check_workspace(const void* workspace, int64_t held, int64_t needed) {
    if (needed == 0) return FSDP_OK;
    if (!workspace || held < needed)
        return fail(FSDP_ERR_INVALID, "the workspace holds %lld bytes, %lld are needed", (long long)(workspace ? held : 0),
                    (long long)needed);
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return fail(FSDP_ERR_ALIGN, "workspace is not 256-byte aligned");
    return FSDP_OK;
}

}  // namespace fsdp_block

extern "C" const char* fsdp_block_last_error(void) { return fsdp_block::t_text; }
