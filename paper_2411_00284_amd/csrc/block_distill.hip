// Distillation from a teacher's top logits: loss and gradient
// (include/fsdp_block.h).
//
// Bound by HBM: a row of logits is read for its maximum and sum (kept running
// together, in one pass) and again for its gradient; the second read comes
// from cache.  A workgroup takes a row; the teacher's entries, at most 1024,
// lie in LDS.

#include "block_device.h"
#include "block_host.h"

#include <algorithm>
#include <cfloat>

namespace fsdp_block {
namespace {

struct DistillArgs {
    const void *logits, *teacher, *ids;
    const float *teacher_lse, *dloss, *lse_in;
    float *loss, *lse;
    void* dlogits;
    int64_t logits_stride, dlogits_stride, tokens;
    int vocab, top, teacher_dtype, ids_64;
    float tau;
};

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float teacher_at(const DistillArgs& a, int64_t i) {
    if (a.teacher_dtype == FSDP_DTYPE_BF16) return float(static_cast<const bf16*>(a.teacher)[i]);
    if (a.teacher_dtype == FSDP_DTYPE_F16) return float(static_cast<const f16*>(a.teacher)[i]);
    return static_cast<const float*>(a.teacher)[i];
}

// An id as the kernel takes it: < 0 no entry, >= vocab out of range.
__device__ __forceinline__ int id_at(const DistillArgs& a, int64_t i) {
    if (!a.ids_64) return static_cast<const int32_t*>(a.ids)[i];
    const int64_t id = static_cast<const int64_t*>(a.ids)[i];
    return id < 0 ? -1 : id > INT32_MAX ? INT32_MAX : int(id);
}

// The running maximum m and sum of 2^((s - m) c) of a softmax.  A maximum of
// -inf counts as 0 in the exponents, so that rows and threads that hold nothing
// but -inf (or nothing) keep a sum of 0.
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void join_softmax(float& m, float& s, float m2, float s2, float c) {
    const float top = fmaxf(m, m2), z = shift_of(top);
    s = s * exp2f((m - z) * c) + s2 * exp2f((m2 - z) * c);
    m = top;
}

template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_kernel(const DistillArgs a) {
    constexpr int kWaves = kThreads / 64;
    __shared__ float p[FSDP_DISTILL_MAX_TOP], picked[FSDP_DISTILL_MAX_TOP];
    __shared__ int ids[FSDP_DISTILL_MAX_TOP];
    __shared__ float wm[kWaves], ws[kWaves];
    __shared__ double wd[kWaves];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const float c = kLog2e / a.tau;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* s = static_cast<const T*>(a.logits) + row * a.logits_stride;
        T* ds = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
        // The teacher's softmax.
        float top = -INFINITY;
        int bad = 0;
        for (int k = t; k < a.top; k += kThreads) {
            const int id = id_at(a, row * a.top + k);
            const float v = id < 0 ? -INFINITY : teacher_at(a, row * a.top + k);
            ids[k] = id;
            p[k] = v;
            picked[k] = id >= 0 && id < a.vocab ? float(s[id]) : 0.f;
            bad |= id >= a.vocab;
            top = v != v || top != top ? NAN : fmaxf(top, v);
        }
        top = __any(top != top) ? NAN : wave_max(top);
        if (lane == 0) wm[wave] = top;
        bad = __syncthreads_or(bad);
        for (int w = 0; w < kWaves; ++w) top = wm[w] != wm[w] || top != top ? NAN : fmaxf(top, wm[w]);
        const bool none = top == -INFINITY;                     // no entry, or none with any mass
        const float scale = a.dlogits ? a.dloss[row] * a.tau : 0.f;
        if (none || bad) {
            const float fill = bad ? NAN : 0.f;
            if (t == 0 && a.loss) a.loss[row] = fill;
            if (t == 0 && a.lse) a.lse[row] = 0.f;
            if (a.dlogits)
                for (int j = t; j < a.vocab; j += kThreads) ds[j] = T(fill);
            __syncthreads();                                    // LDS is the next row's
            continue;
        }
        float one[1] = {0.f};
        for (int k = t; k < a.top; k += kThreads) one[0] += exp2f((p[k] - top) * c);
        group_sum<kThreads, 1>(one, ws);
        const double teacher_lse = a.teacher_lse ? double(a.teacher_lse[row]) : double(top) / double(a.tau) + log(double(one[0]));
        // The student's softmax.
        double lse;
        if (a.lse_in) {
            lse = double(a.lse_in[row]);
        } else {
            float m = -INFINITY, sum = 0.f;
            for (int j = t * 8; j < a.vocab; j += kThreads * 8) {
                const int left = a.vocab - j;
                const Eight<T> v = load_some(s + j, left);
                float most = float(v[0]);
#pragma unroll
                for (int i = 1; i < 8; ++i)
                    if (i < left) most = fmaxf(most, float(v[i]));
                const float next = fmaxf(m, most), z = shift_of(next);
                sum *= exp2f((m - z) * c);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) sum += exp2f((float(v[i]) - z) * c);
                m = next;
            }
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) join_softmax(m, sum, __shfl_xor(m, d), __shfl_xor(sum, d), c);
            __syncthreads();                                    // ws has been read
            if (lane == 0) {
                wm[wave] = m;
                ws[wave] = sum;
            }
            __syncthreads();
            m = -INFINITY;
            sum = 0.f;
            for (int w = 0; w < kWaves; ++w) join_softmax(m, sum, wm[w], ws[w], c);
            lse = double(m) / double(a.tau) + log(double(sum));
        }
        if (t == 0 && a.lse) a.lse[row] = float(lse);
        // p_k, their sum and the loss.
        const float shift = float(teacher_lse * double(a.tau) - double(top));      // p_k = exp((v_k - top - shift) / tau)
        float mass = 0.f;
        double loss = 0.0;
        for (int k = t; k < a.top; k += kThreads) {
            const float v = p[k], pk = exp2f(((v - top) - shift) * c);
            mass += pk;
            p[k] = pk;
            if (pk != 0.f) loss += double(pk) * ((double(v) - double(picked[k])) / double(a.tau) - (teacher_lse - lse));
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            mass += __shfl_xor(mass, d);
            loss += __shfl_xor(loss, d);
        }
        __syncthreads();
        if (lane == 0) {
            ws[wave] = mass;
            wd[wave] = loss;
        }
        __syncthreads();
        mass = 0.f;
        loss = 0.0;
        for (int w = 0; w < kWaves; ++w) {
            mass += ws[w];
            loss += wd[w];
        }
        if (t == 0 && a.loss) a.loss[row] = float(double(a.tau) * double(a.tau) * loss);
        if (a.dlogits) {
            // q = exp((s - base - rest) / tau): the logsumexp in two parts, so that
            // logits far from 0 lose nothing.
            const float base = float(lse * double(a.tau)), rest = float(lse * double(a.tau) - double(base));
            const bool zero = a.dloss[row] == 0.f;
            for (int j = t * 8; j < a.vocab; j += kThreads * 8) {
                const Eight<T> v = load_some(s + j, a.vocab - j);
                float out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = zero ? 0.f : scale * mass * exp2f(((float(v[i]) - base) - rest) * c);
                store_some(ds + j, a.vocab - j, out);
            }
            __syncthreads();                                    // the entries' places are written again
            if (!zero)
                for (int k = t; k < a.top; k += kThreads) {
                    if (ids[k] < 0) continue;
                    float same = 0.f;
                    for (int i = 0; i < a.top; ++i) same += ids[i] == ids[k] ? p[i] : 0.f;
                    ds[ids[k]] = T(scale * (mass * exp2f(((picked[k] - base) - rest) * c) - same));
                }
        }
        __syncthreads();                                        // LDS is the next row's
    }
}

fsdp_status run(const fsdp_distill_args* args, bool backward, hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_distill_args& a = *args;
    if (a.tokens < 0) return fail(FSDP_ERR_INVALID, "tokens is negative");
    if (a.vocab < 1 || a.top < 1) return fail(FSDP_ERR_INVALID, "vocab and top must be at least 1");
    if (a.vocab > INT32_MAX - (1 << 16)) return fail(FSDP_ERR_OVERFLOW, "vocab does not fit 31 bits");
    if (a.top > FSDP_DISTILL_MAX_TOP) return fail(FSDP_ERR_TOO_MANY, "top is above %d", FSDP_DISTILL_MAX_TOP);
    if (!known_dtype(a.dtype) || !known_dtype(a.teacher_dtype)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (a.ids_64 != 0 && a.ids_64 != 1) return fail(FSDP_ERR_INVALID, "ids_64 must be 0 or 1");
    if (!(a.temperature > 0.f) || !__builtin_isfinite(a.temperature))
        return fail(FSDP_ERR_INVALID, "temperature must be positive and finite");
    if (backward && a.tokens > 0 && (!a.lse || !a.dlogits)) return fail(FSDP_ERR_INVALID, "lse and dlogits are needed");
    if (!backward && a.tokens > 0 && !a.loss && !a.lse && !a.dlogits) return fail(FSDP_ERR_INVALID, "no output is wanted");
    const int64_t t = a.tokens;
    Checked m;
    m.add("logits", a.logits, t, a.vocab, a.logits_stride, a.dtype, true);
    m.add("teacher", a.teacher, t, a.top, a.top, a.teacher_dtype, true);
    // int64 ids: twice as many fp32-sized elements
    m.add("ids", a.ids, t, a.top << a.ids_64, a.top << a.ids_64, FSDP_DTYPE_F32, true);
    if (a.ids && a.ids_64 && reinterpret_cast<uintptr_t>(a.ids) % 8 != 0) return fail(FSDP_ERR_ALIGN, "ids is not element-aligned");
    m.add_vector("teacher_lse", a.teacher_lse, t, FSDP_DTYPE_F32, false);
    m.add_vector("dloss", a.dloss, t, FSDP_DTYPE_F32, a.dlogits);
    if (!backward) m.add_vector("loss", a.loss, t, FSDP_DTYPE_F32, false, true);
    m.add_vector("lse", a.lse, t, FSDP_DTYPE_F32, false, !backward);
    m.add("dlogits", a.dlogits, t, a.vocab, a.dlogits_stride, a.dtype, false, true, a.logits);
    const fsdp_status st = m.done();
    if (st != FSDP_OK || t == 0) return st;
    const DistillArgs k{a.logits, a.teacher, a.ids, a.teacher_lse, a.dloss, backward ? a.lse : nullptr,
                        backward ? nullptr : a.loss, backward ? nullptr : a.lse, a.dlogits, a.logits_stride,
                        a.dlogits_stride, t, int(a.vocab), int(a.top), a.teacher_dtype, a.ids_64, a.temperature};
    const dim3 grid(unsigned(std::min<int64_t>(t, int64_t(1) << 21)));
    const auto of = [&](auto type) {
        using T = decltype(type);
        return a.vocab <= 8192 ? launch(distill_kernel<T, 256>, k, grid, 256, stream)
                               : launch(distill_kernel<T, 1024>, k, grid, 1024, stream);
    };
    return a.dtype == FSDP_DTYPE_BF16 ? of(bf16(0.f)) : a.dtype == FSDP_DTYPE_F16 ? of(f16(0.f)) : of(0.f);
}

}  // namespace
}  // namespace fsdp_block

extern "C" fsdp_status fsdp_block_distill(const fsdp_distill_args* args, hipStream_t stream) {
    return fsdp_block::run(args, false, stream);
}

extern "C" fsdp_status fsdp_block_distill_grad(const fsdp_distill_args* args, hipStream_t stream) {
    return fsdp_block::run(args, true, stream);
}
