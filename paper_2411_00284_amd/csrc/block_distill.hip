// Distillation from a teacher's top logits: loss and gradient
// (include/fsdp_block.h).
//
// Bound by HBM: a row of logits is read for its maximum and sum (kept running
// together, in one pass), and again for its gradient; a workgroup takes a row
// and holds what it can of it in registers, so that the second read is of the
// rest only, from cache.  Loss and gradient of 4096 x 128256 in bf16 take 440 us
// (4.8 TB/s of one read and one write).  The teacher's entries, at most 1024, lie
// in LDS.

#include "block_device.h"
#include "block_host.h"
#include "block_softmax.h"

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

// f(entry, sum of p over the entries with its id).  Repeated ids are found
// in LDS: an entry that is alone in its slot of a table is no repeat, others are
// put into another table, and what still shares a slot after kRounds looks at
// all entries.  (All pairs at once: 160 us of 660 at 4096 rows of 512 entries; six tables leave
// hardly one of 1024 different ids to the last step.)
constexpr int kSlots = 2048, kRounds = 6, kFewEntries = 16;
template <int kThreads, typename F>
__device__ __forceinline__ void for_same_ids(int top, const int* ids, const float* p, int* slots, F f) {
    constexpr int kEntries = FSDP_DISTILL_MAX_TOP / kThreads;
    uint32_t open = ~0u;                         // a bit per entry of this thread
    if (top > kFewEntries) {
        for (int round = 0; round < kRounds; ++round) {
            for (int i = threadIdx.x; i < kSlots; i += kThreads) slots[i] = 0;
            __syncthreads();
            const unsigned mix = 2654435761u + 2246822518u * unsigned(round);       // odd: a table of its own
            const auto slot = [&](int k) { return &slots[unsigned(ids[k]) * mix >> 21]; };
            const auto is_open = [&](int e, int k) { return k < top && ids[k] >= 0 && (open >> e & 1); };
#pragma unroll
            for (int e = 0; e < kEntries; ++e)
                if (const int k = int(threadIdx.x) + e * kThreads; is_open(e, k)) atomicAdd(slot(k), 1);
            __syncthreads();
            uint32_t still = 0;
#pragma unroll
            for (int e = 0; e < kEntries; ++e)
                if (const int k = int(threadIdx.x) + e * kThreads; is_open(e, k) && *slot(k) > 1) still |= 1u << e;
            open = still;
            if (!__syncthreads_or(int(open))) break;
        }
    }
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        const int k = int(threadIdx.x) + e * kThreads;
        if (k >= top || ids[k] < 0) continue;
        float same = p[k];
        if (open >> e & 1) {
            const int id = ids[k];
            same = 0.f;
            for (int i = 0; i < top; ++i) same += ids[i] == id ? p[i] : 0.f;
        }
        f(k, same);
    }
}

// kHeld units per thread stay in registers; those of the first group are asked
// for before the teacher's entries are looked at.
template <typename T, int kThreads, int kHeld>
__global__ __launch_bounds__(kThreads, kHeld > 4 ? 4 : 5) void distill_kernel(const DistillArgs a) {
    constexpr int kWaves = kThreads / 64, n = Unit<T>::n;
    static_assert(kHeld >= 4 && kHeld % 2 == 0);
    __shared__ float p[FSDP_DISTILL_MAX_TOP], picked[FSDP_DISTILL_MAX_TOP];
    __shared__ int ids[FSDP_DISTILL_MAX_TOP], slots[kSlots];
    __shared__ float wm[kWaves], ws[kWaves], wt[kWaves], wp[kWaves];
    __shared__ double wd[kWaves];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, vocab = a.vocab, units = vocab / n;
    const int single = units * n + t;                           // this thread's element after the units
    const float c = fminf(kLog2e / a.tau, FLT_MAX);             // finite for a subnormal tau: 0 c is 0
    const double tau = double(a.tau), per_tau = 1.0 / tau, ln2 = 0.6931471805599453;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* const s = static_cast<const T*>(a.logits) + row * a.logits_stride;
        T* const ds = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
        const float weight = a.dlogits ? a.dloss[row] : 0.f;
        Unit<T> held[kHeld / 2][2];
#pragma unroll
        for (int u = 0; u < 4; ++u) held[u / 2][u % 2].load(s, t + u * kThreads, units);
        const float lone = single < vocab ? float(s[single]) : -INFINITY;
        // The teacher's entries: id, logit, the student's logit there (which an in-place gradient overwrites).
        // Each is its thread's own, from here to the end.
        float top = -INFINITY;
        int bad = 0;
        for (int k = t; k < a.top; k += kThreads) {
            const int id = id_at(a, row * a.top + k);
            const float v = id < 0 ? -INFINITY : teacher_at(a, row * a.top + k);
            ids[k] = id;
            p[k] = v;
            picked[k] = id >= 0 && id < vocab ? float(s[id]) : 0.f;
            bad |= id >= vocab;
            top = v != v || top != top ? NAN : fmaxf(top, v);
        }
        top = __any(top != top) ? NAN : wave_max(top);
        if (lane == 0) wm[wave] = top;
        bad = __syncthreads_or(bad);
        top = wm[lane % kWaves];                                // over the waves, as over a wave's lanes
        top = __any(top != top) ? NAN : wave_max(top);
        if (top == -INFINITY || bad) {                          // no entry with any mass, or one out of range
            const float fill = bad ? NAN : 0.f;
            if (t == 0 && a.loss) a.loss[row] = fill;
            if (t == 0 && a.lse) a.lse[row] = 0.f;
            if (a.dlogits) {
                for (int u = t; u < units; u += kThreads) Unit<T>::store(ds, u, typename Unit<T>::vec(T(fill)));
                if (single < vocab) ds[single] = T(fill);
            }
            __syncthreads();                                    // LDS is the next row's
            continue;
        }
        // What depends on the entries alone is left to the waves that hold some.
        const bool some = wave * 64 < a.top;
        float sum = 0.f;
        if (some) {
            for (int k = t; k < a.top; k += kThreads) sum += exp2_fast((p[k] - top) * c);
            sum = wave_sum(sum);
        }
#pragma unroll
        for (int u = 4; u < kHeld; ++u) held[u / 2][u % 2].load(s, t + u * kThreads, units);
        Softmax x;
        if (!a.lse_in) {
#pragma unroll
            for (int u = 0; u < kHeld / 2; ++u) add_units(x, held[u], c);
            for (int j = t + kHeld * kThreads; j < units; j += kTogether * kThreads) {
                Unit<T> u[kTogether];
#pragma unroll
                for (int k = 0; k < kTogether; ++k) u[k].load(s, j + k * kThreads, units);
                add_units(x, u, c);
            }
            x.join(lone, lone == -INFINITY ? 0.f : 1.f, c);
            // Over the wave: the maximum first, then sums of one shift.
            const float m = wave_max(x.m);
            x.s = wave_sum(Softmax::moved(x.s, x.m, Softmax::base(m), c));
            x.m = m;
        }
        __syncthreads();                                        // wm has been read
        if (lane == 0) {
            wt[wave] = sum;
            wm[wave] = x.m;
            ws[wave] = x.s;
        }
        __syncthreads();
        sum = wave_sum(lane < kWaves ? wt[lane] : 0.f);
        if (!a.lse_in) {
            const float m = wm[lane % kWaves];
            x.m = wave_max(m);
            x.s = wave_sum(lane < kWaves ? Softmax::moved(ws[lane], m, Softmax::base(x.m), c) : 0.f);
        }
        // Both logarithms as log sums over their maxima, apart from these: of rows of one mask
        // value the sum would be lost beside it.
        const double log_sum = log2_of(x.s) * ln2;
        if (t == 0 && a.lse) a.lse[row] = float(double(x.m) * per_tau + log_sum);
        // p_k = exp((v_k - top) / tau - over) = exp((v_k - top - rest) / tau), their sum and the loss.
        const double over = a.teacher_lse ? double(a.teacher_lse[row]) - double(top) * per_tau : log2_of(sum) * ln2;
        const float rest = float(over * tau);
        float mass = 0.f;
        double loss = 0.0;
        if (some) {
            for (int k = t; k < a.top; k += kThreads) {
                const float v = p[k], pk = exp2_fast(((v - top) - rest) * c);
                mass += pk;
                // log p - log q
                if (pk != 0.f)
                    loss += double(pk) * (((double(v) - double(top)) * per_tau - over) -
                                          ((double(picked[k]) - double(x.m)) * per_tau - log_sum));
                p[k] = pk;
            }
            mass = wave_sum(mass);
            if (a.loss)
#pragma unroll
                for (int d = 32; d > 0; d >>= 1) loss += __shfl_xor(loss, d);
        }
        if (lane == 0) {
            wp[wave] = mass;
            wd[wave] = loss;
        }
        __syncthreads();
        if (wave == 0 && a.loss) {
            loss = lane < kWaves ? wd[lane] : 0.0;
#pragma unroll
            for (int d = kWaves / 2; d > 0; d >>= 1) loss += __shfl_xor(loss, d);
            if (t == 0) a.loss[row] = float(tau * tau * loss);
        }
        if (a.dlogits) {
            mass = wave_sum(lane < kWaves ? wp[lane] : 0.f);
            // q = 2^((s - base) c) times what its base leaves: the sum over the row's maximum, or
            // of a saved lse what float(lse tau) misses of it.
            const float scale = weight * a.tau;
            const bool zero = weight == 0.f;
            float base = Softmax::base(x.m), factor = scale * mass / x.s;
            if (a.lse_in) {
                const double b = double(a.lse_in[row]) * tau;
                base = b > FLT_MAX ? FLT_MAX : b < -FLT_MAX ? -FLT_MAX : float(b);
                factor = scale * mass * exp2_fast(float((double(base) - b) * double(c)));
            }
            const auto slope = [&](float v) { return T(zero ? 0.f : factor * exp2_fast((v - base) * c)); };
            const auto put = [&](const Unit<T>& u, int unit) {
                if (unit >= units) return;
                typename Unit<T>::vec out;
#pragma unroll
                for (int i = 0; i < n; ++i) out[i] = slope(float(u.v[i]));
                Unit<T>::store(ds, unit, out);
            };
#pragma unroll
            for (int u = 0; u < kHeld; ++u) put(held[u / 2][u % 2], t + u * kThreads);
            for (int j = t + kHeld * kThreads; j < units; j += kTogether * kThreads) {
                Unit<T> u[kTogether];
#pragma unroll
                for (int k = 0; k < kTogether; ++k) u[k].template load<true>(s, j + k * kThreads, units);
#pragma unroll
                for (int k = 0; k < kTogether; ++k) put(u[k], j + k * kThreads);
            }
            if (single < vocab) ds[single] = slope(lone);
            __syncthreads();                                    // the entries' places are written again
            if (!zero)                                          // the same for the whole workgroup
                for_same_ids<kThreads>(a.top, ids, p, slots, [&](int k, float same) {
                    ds[ids[k]] = T(factor * exp2_fast((picked[k] - base) * c) - scale * same);
                });
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
    m.add_in_place("logits", a.logits, t, a.vocab, a.logits_stride, a.dtype, true);
    m.add_in_place("teacher", a.teacher, t, a.top, a.top, a.teacher_dtype, true);
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
    fsdp_status found = FSDP_OK;
    const int cus = cu_count(&found);
    if (cus == 0) return found;
    // Rows that 256 threads hold in four units each: the fewest steps from one
    // wave to the next.  Few rows: as many threads as a workgroup has, each with
    // more of the row on its way at once.  Else 256 threads, the most workgroups
    // that a row's chain of loads and sums can hide behind; for a row that is read
    // twice and long, 512, which hold twice of it (at 4096 x 128256 in bf16, loss
    // and gradient: 445 instead of 488 us; the loss alone 210 instead of 191, and at
    // 8192 x 32000 both 247 instead of 224).
    const int64_t units = ceil_div(a.vocab, 16 / elem_bytes(a.dtype));
    const bool twice = !backward && a.dlogits;
    const auto of = [&](auto type) {
        using T = decltype(type);
        if (units <= 4 * 256) return launch(distill_kernel<T, 256, 4>, k, grid, 256, stream);
        if (t <= cus) return launch(distill_kernel<T, 1024, 8>, k, grid, 1024, stream);
        if (!twice || units <= 4096) return launch(distill_kernel<T, 256, 8>, k, grid, 256, stream);
        return launch(distill_kernel<T, 512, 8>, k, grid, 512, stream);
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
