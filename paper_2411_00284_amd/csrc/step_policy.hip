// Clipped policy loss of sampled tokens with its KL term: loss and gradient
// (include/fsdp_step.h).
//
// Bound by HBM: a row of logits is read for its maximum and sum (kept running
// together, in one pass), and again for its gradient; a workgroup takes a row and
// holds what it can of it in registers, so that the second read is of the rest only,
// from cache.  Rows of masked tokens are not read at all, and rows whose gradient is
// zero (past the clip, without a KL term) are not read again.
//
// 4096 x 128256 in bf16 with the gradient takes 413 us, 5.1 TB/s of one read and one
// write; 1531 x 50257 in fp16 from a saved logsumexp 63 us with three rows in ten masked, 4.2 TB/s.

#include "block_device.h"
#include "block_host.h"
#include "block_softmax.h"
#include "fsdp_step.h"

#include <algorithm>
#include <cfloat>

namespace fsdp_block {
namespace {

struct PolicyArgs {
    const void *logits, *actions;
    const float *old_logp, *advantages, *ref_logp, *dloss, *lse_in;
    float *loss, *logp, *lse;
    void* dlogits;
    int64_t logits_stride, dlogits_stride, tokens;
    int vocab, actions_64;
    float low, high, kl, tau;
};

// exp(d) - d - 1, with no difference of nearly equal numbers: its series near 0.
__device__ __forceinline__ float kl_of(float d) {
    if (fabsf(d) < 0.5f) {
        float p = 1.f / 362880.f;                // d^2 (1/2 + d/6 + ... + d^7/9!): the rest is below 2^-24 of it
#pragma unroll
        for (int i = 8; i >= 2; --i) {
            constexpr float inverse[9] = {0.f, 0.f, 1.f / 2, 1.f / 6, 1.f / 24, 1.f / 120, 1.f / 720, 1.f / 5040, 1.f / 40320};
            p = fmaf(p, d, inverse[i]);
        }
        return d * d * p;
    }
    return d == INFINITY ? d : expm1f(d) - d;
}

// A token's loss, and its slope with respect to logp. The differences of logarithms are
// 64-bit ones; from there on 32 bits keep all that their own errors leave (with exp and
// expm1 in 64 bits the rows' registers would go to memory and back).
__device__ __forceinline__ void token_loss(const PolicyArgs& a, int64_t row, double logp, float& loss, float& slope) {
    const float adv = a.advantages[row], r = expf(float(logp - double(a.old_logp[row])));
    // A token without advantage has no part of it, whatever its ratio.
    const float gain = adv == 0.f ? 0.f : r * adv;
    const float clipped = adv == 0.f ? 0.f : fminf(fmaxf(r, 1.f - a.low), 1.f + a.high) * adv;
    const bool flat = gain > clipped;            // a NaN is not
    loss = flat ? -clipped : -gain;
    slope = flat ? 0.f : -gain;
    if (a.ref_logp && a.kl != 0.f) {
        const float d = float(double(a.ref_logp[row]) - logp);
        loss = fmaf(a.kl, kl_of(d), loss);
        slope = fmaf(-a.kl, expm1f(d), slope);
    }
}

// A saved lse is rounded to 32 bits, and q and the ratio are off by exp of its rounding: by 2^-11 of
// themselves below 2^14. From there on (small temperatures, rows far from 0 or all at a mask's finite
// value) the row's maximum and sum are taken again, which costs another pass over the row: 77 us instead of
// 66 at 1531 x 50257 in fp16.
constexpr float kSavedLse = 16384.f;

// kHeld units per thread stay in registers, the others are streamed kStream at a time.
constexpr int kStream = 4;
template <typename T, int kThreads, int kHeld>
__global__ __launch_bounds__(kThreads, kHeld > 4 ? 4 : 5) void policy_kernel(const PolicyArgs a) {
    constexpr int kWaves = kThreads / 64, n = Unit<T>::n;
    static_assert(kHeld >= 4 && kHeld % 2 == 0);
    __shared__ float wm[kWaves], ws[kWaves];
    __shared__ float weight_of, at_action;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, vocab = a.vocab, units = vocab / n;
    const int single = units * n + t;                           // this thread's element after the units
    const float c = fminf(kLog2e / a.tau, FLT_MAX);             // finite for the smallest tau: 0 c is 0
    const double per_tau = 1.0 / double(a.tau), ln2 = 0.6931471805599453;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* const s = static_cast<const T*>(a.logits) + row * a.logits_stride;
        T* const ds = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
        const int64_t action = a.actions_64 ? static_cast<const int64_t*>(a.actions)[row] : static_cast<const int32_t*>(a.actions)[row];
        const auto fill = [&](float v) {
            if (!a.dlogits) return;
            for (int u = t; u < units; u += kThreads) Unit<T>::store(ds, u, typename Unit<T>::vec(T(v)));
            if (single < vocab) ds[single] = T(v);
        };
        if (action < 0 || action >= vocab) {                    // masked, or out of range
            const float v = action < 0 ? 0.f : NAN;
            if (t == 0 && a.loss) a.loss[row] = v;
            if (t == 0 && a.logp) a.logp[row] = v;
            if (t == 0 && a.lse) a.lse[row] = v;
            fill(v != 0.f && a.dlogits && a.dloss[row] == 0.f ? 0.f : v);
            continue;
        }
        const float picked = float(s[action]);                  // before an in-place gradient overwrites it
        const bool gradient = a.dlogits && a.dloss[row] != 0.f, whole = !a.lse_in || gradient;
        const bool saved = a.lse_in && fabsf(a.lse_in[row]) < kSavedLse;   // not a NaN
        Unit<T> held[kHeld / 2][2];
        float lone = -INFINITY;
        Softmax x;
        if (whole) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u) held[u / 2][u % 2].load(s, t + u * kThreads, units);
            lone = single < vocab ? float(s[single]) : -INFINITY;
        }
        if (whole && !saved) {
#pragma unroll
            for (int u = 0; u < kHeld / 2; ++u) add_units(x, held[u], c);
            for (int j = t + kHeld * kThreads; j < units; j += kStream * kThreads) {
                Unit<T> u[kStream];
#pragma unroll
                for (int k = 0; k < kStream; ++k) u[k].load(s, j + k * kThreads, units);
                add_units(x, u, c);
            }
            x.join(lone, lone == -INFINITY ? 0.f : 1.f, c);
            // Over the wave, and the waves: the maximum first, then sums of one shift.
            const float m = wave_max(x.m);
            x.s = wave_sum(Softmax::moved(x.s, x.m, Softmax::base(m), c));
            x.m = m;
            if (lane == 0) {
                wm[wave] = x.m;
                ws[wave] = x.s;
            }
            __syncthreads();
            const float mine = wm[lane % kWaves];
            x.m = wave_max(mine);
            x.s = wave_sum(lane < kWaves ? Softmax::moved(ws[lane], mine, Softmax::base(x.m), c) : 0.f);
        }
        if (wave == 0) {                                        // every lane the same
            const double log_sum = saved ? 0.0 : log2_of(x.s) * ln2;
            // The difference to the maximum first: a row of one mask value would lose the sum beside it.
            const double logp = saved ? double(picked) * per_tau - double(a.lse_in[row]) : (double(picked) - double(x.m)) * per_tau - log_sum;
            float loss, slope;
            token_loss(a, row, logp, loss, slope);
            const float weight = gradient ? float(double(a.dloss[row]) * double(slope) * per_tau) : 0.f;
            const float action_slope = weight * -expm1f(float(logp));      // 1 - q, with no difference of the two
            if (lane == 0) {
                if (a.loss) a.loss[row] = loss;
                if (a.logp) a.logp[row] = float(logp);
                if (a.lse) a.lse[row] = float(double(x.m) * per_tau + log_sum);
                weight_of = weight;
                at_action = action_slope;
            }
        }
        if (!a.dlogits) {
            __syncthreads();                                    // LDS is the next row's
            continue;
        }
        __syncthreads();
        const float weight = weight_of;
        if (weight == 0.f) {
            fill(0.f);
        } else {
            // q = 2^((s - base) c) times what its base leaves: the sum over the row's maximum, or
            // of a saved lse what float(lse tau) misses of it.
            float base = Softmax::base(x.m), factor = -weight / x.s;
            if (saved) {
                const double b = double(a.lse_in[row]) * double(a.tau);
                base = b > FLT_MAX ? FLT_MAX : b < -FLT_MAX ? -FLT_MAX : float(b);
                factor = -weight * exp2_fast(float((double(base) - b) * double(c)));
            }
            const auto slope = [&](float v) { return T(factor * exp2_fast((v - base) * c)); };
            const auto put = [&](const Unit<T>& u, int unit) {
                if (unit >= units) return;
                typename Unit<T>::vec out;
#pragma unroll
                for (int i = 0; i < n; ++i) out[i] = slope(float(u.v[i]));
                // The action's element in its place: no store that another one would have to follow.
                if (const int i = int(action) - unit * n; i >= 0 && i < n) {
                    const T v = T(at_action);
#pragma unroll
                    for (int k = 0; k < n; ++k) out[k] = k == i ? v : out[k];
                }
                Unit<T>::store(ds, unit, out);
            };
#pragma unroll
            for (int u = 0; u < kHeld; ++u) put(held[u / 2][u % 2], t + u * kThreads);
            for (int j = t + kHeld * kThreads; j < units; j += kStream * kThreads) {
                Unit<T> u[kStream];
#pragma unroll
                for (int k = 0; k < kStream; ++k) u[k].template load<true>(s, j + k * kThreads, units);
#pragma unroll
                for (int k = 0; k < kStream; ++k) put(u[k], j + k * kThreads);
            }
            if (single < vocab) ds[single] = single == action ? T(at_action) : slope(lone);
        }
        __syncthreads();                                        // LDS is the next row's
    }
}

fsdp_status run(const fsdp_step_policy_args* args, bool backward, hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_step_policy_args& a = *args;
    if (a.tokens < 0) return fail(FSDP_ERR_INVALID, "tokens is negative");
    if (a.vocab < 1) return fail(FSDP_ERR_INVALID, "vocab must be at least 1");
    if (a.vocab > INT32_MAX - (1 << 16)) return fail(FSDP_ERR_OVERFLOW, "vocab does not fit 31 bits");
    if (!known_dtype(a.dtype)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (a.actions_64 != 0 && a.actions_64 != 1) return fail(FSDP_ERR_INVALID, "actions_64 must be 0 or 1");
    // A gradient is of the size of 1 / temperature.
    if (!(a.temperature >= FLT_MIN) || !__builtin_isfinite(a.temperature))
        return fail(FSDP_ERR_INVALID, "temperature must be positive, normal and finite");
    if (!(a.clip_low >= 0.f) || a.clip_low > 1.f) return fail(FSDP_ERR_INVALID, "clip_low must be in 0 .. 1");
    if (!(a.clip_high >= 0.f)) return fail(FSDP_ERR_INVALID, "clip_high must not be negative");
    if (!__builtin_isfinite(a.kl_weight)) return fail(FSDP_ERR_INVALID, "kl_weight must be finite");
    const int64_t t = a.tokens;
    if (t > 0 && a.kl_weight != 0.f && !a.ref_logp) return fail(FSDP_ERR_INVALID, "kl_weight needs ref_logp");
    if (backward && t > 0 && (!a.lse || !a.dlogits)) return fail(FSDP_ERR_INVALID, "lse and dlogits are needed");
    if (!backward && t > 0 && !a.loss && !a.logp && !a.lse && !a.dlogits) return fail(FSDP_ERR_INVALID, "no output is wanted");
    Checked m;
    m.add_in_place("logits", a.logits, t, a.vocab, a.logits_stride, a.dtype, true);
    // int64 actions: twice as many elements of four bytes
    m.add("actions", a.actions, t > 0 ? 1 : 0, t << a.actions_64, t << a.actions_64, FSDP_DTYPE_F32, true);
    if (a.actions && a.actions_64 && reinterpret_cast<uintptr_t>(a.actions) % 8 != 0)
        return fail(FSDP_ERR_ALIGN, "actions is not element-aligned");
    m.add_vector("old_logp", a.old_logp, t, FSDP_DTYPE_F32, true);
    m.add_vector("advantages", a.advantages, t, FSDP_DTYPE_F32, true);
    m.add_vector("ref_logp", a.ref_logp, t, FSDP_DTYPE_F32, false);
    m.add_vector("dloss", a.dloss, t, FSDP_DTYPE_F32, a.dlogits);
    if (!backward) m.add_vector("loss", a.loss, t, FSDP_DTYPE_F32, false, true);
    if (!backward) m.add_vector("logp", a.logp, t, FSDP_DTYPE_F32, false, true);
    m.add_vector("lse", a.lse, t, FSDP_DTYPE_F32, false, !backward);
    m.add("dlogits", a.dlogits, t, a.vocab, a.dlogits_stride, a.dtype, false, true, a.logits);
    const fsdp_status st = m.done();
    if (st != FSDP_OK || t == 0) return st;
    const PolicyArgs k{a.logits, a.actions, a.old_logp, a.advantages, a.ref_logp, a.dloss, backward ? a.lse : nullptr,
                       backward ? nullptr : a.loss, backward ? nullptr : a.logp, backward ? nullptr : a.lse, a.dlogits,
                       a.logits_stride, a.dlogits_stride, t, int(a.vocab), a.actions_64, a.clip_low, a.clip_high, a.kl_weight,
                       a.temperature};
    const dim3 grid(unsigned(std::min<int64_t>(t, int64_t(1) << 21)));
    fsdp_status found = FSDP_OK;
    const int cus = cu_count(&found);
    if (cus == 0) return found;
    // A wave that holds a row whole: no wait between waves (6669 x 1847 in bf16, loss and gradient:
    // 19.1 us instead of 29.5). Else as the distillation loss, whose passes over the logits are the
    // same: few rows, 1024 threads; 256, or 512 for a long row that is read twice.
    const int64_t units = ceil_div(a.vocab, 16 / elem_bytes(a.dtype));
    const bool twice = !backward && a.dlogits;
    const auto of = [&](auto type) {
        using T = decltype(type);
        if (units <= 8 * 64) return launch(policy_kernel<T, 64, 8>, k, grid, 64, stream);
        if (units <= 4 * 256) return launch(policy_kernel<T, 256, 4>, k, grid, 256, stream);
        if (t <= cus) return launch(policy_kernel<T, 1024, 8>, k, grid, 1024, stream);
        if (!twice || units <= 4096) return launch(policy_kernel<T, 256, 8>, k, grid, 256, stream);
        return launch(policy_kernel<T, 512, 8>, k, grid, 512, stream);
    };
    return a.dtype == FSDP_DTYPE_BF16 ? of(bf16(0.f)) : a.dtype == FSDP_DTYPE_F16 ? of(f16(0.f)) : of(0.f);
}

}  // namespace
}  // namespace fsdp_block

extern "C" fsdp_status fsdp_step_policy(const fsdp_step_policy_args* args, hipStream_t stream) {
    return fsdp_block::run(args, false, stream);
}

extern "C" fsdp_status fsdp_step_policy_grad(const fsdp_step_policy_args* args, hipStream_t stream) {
    return fsdp_block::run(args, true, stream);
}
