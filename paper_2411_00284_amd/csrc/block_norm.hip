// The norms before and after a block, with the gate and the residual add
// between them, and their gradient (include/fsdp_block.h).
//
// Bound by HBM: a row's elements are read once into registers, eight
// neighbouring ones per thread and chunk, and everything after that (both row
// statistics, the outputs) comes from there.  A row belongs to one team of
// threads: a wave for short rows (four teams in a workgroup, no barrier), a
// workgroup for longer ones.  8192 x 4096 in bf16 takes 55 us (4.9 TB/s); the
// gradient of 8192 x 8192 with an fp32 stream, both weights and a gate 251 us (4.8
// TB/s), 12 of them the join of the column sums.
//
// Loads and stores go through the caches.  Past them (non-temporal) the forward at
// 8192 x 4096 changes by 1 % and loses 25 % at 32768 x 256; an earlier form of the
// gradient went from 99 to 92 us at 8192 x 4096 and from 282 to 238 at 4096 x 16384
// (95 and 230 now, through the caches).

#include "block_device.h"
#include "block_host.h"
#include "block_join.h"

#include <algorithm>

namespace fsdp_block {
namespace {

struct NormArgs {
    const void *x, *branch, *post, *gate, *pre;
    void *y, *h;
    int64_t x_stride, branch_stride, y_stride, h_stride;
    int64_t tokens, group_rows;      // tokens that share a row of the gate
    int hidden;
    float eps, residual_scale, branch_scale;
};

template <typename T>
__device__ __forceinline__ const T* row_of(const void* p, int64_t row, int64_t stride) {
    return static_cast<const T*>(p) + row * stride;
}
template <typename T>
__device__ __forceinline__ T* row_of(void* p, int64_t row, int64_t stride) {
    return static_cast<T*>(p) + row * stride;
}

// Chunk c of a team's thread t starts at element 8 * (c * kTeam + t).
#define FSDP_CHUNKS(c, at, left)                                                     \
    _Pragma("unroll") for (int c = 0; c < kChunks; ++c)                              \
        if (const int at = 8 * (c * kTeam + t), left = hidden - at; left > 0)

template <int kTeam>
constexpr int kTeams = kTeam < 256 ? 256 / kTeam : 1;

template <typename TX, typename TB, typename TW, int kTeam, int kChunks>
__global__ __launch_bounds__(kTeam* kTeams<kTeam>) void norm_kernel(const NormArgs a) {
    __shared__ float part[2][kTeam / 64];
    const int t = threadIdx.x % kTeam;
    const int hidden = a.hidden;
    int flip = 0;
    const auto sum = [&](float v) {
        float one[1] = {v};
        group_sum<kTeam, 1>(one, part[flip]);
        flip ^= 1;
        return one[0];
    };
    for (int64_t row = int64_t(blockIdx.x) * kTeams<kTeam> + threadIdx.x / kTeam; row < a.tokens;
         row += int64_t(gridDim.x) * kTeams<kTeam>) {
        float v[kChunks][8];
        Eight<TX> x[kChunks];
        const TX* from = row_of<TX>(a.x, row, a.x_stride);
        FSDP_CHUNKS(c, at, left) x[c] = load_some(from + at, left);
        if (a.branch) {
            Eight<TB> b[kChunks];
            const TB* branch = row_of<TB>(a.branch, row, a.branch_stride);
            FSDP_CHUNKS(c, at, left) b[c] = load_some(branch + at, left);
            float scale = a.branch_scale;
            if (a.post) {
                float s = 0.f;
                FSDP_CHUNKS(c, at, left)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s += float(b[c][i]) * float(b[c][i]);
                scale *= rsqrtf(sum(s) / float(hidden) + a.eps);
            }
            const TB* gate = a.gate ? row_of<TB>(a.gate, a.group_rows < a.tokens ? row / a.group_rows : 0, hidden) : nullptr;
            FSDP_CHUNKS(c, at, left) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = scale * float(b[c][i]);
                if (a.post) {
                    const Eight<TW> w = load_some(static_cast<const TW*>(a.post) + at, left);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] *= float(w[i]);
                }
                if (gate) {
                    const Eight<TB> g = load_some(gate + at, left);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] *= float(g[i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += a.residual_scale * float(x[c][i]);
            }
        } else {
            FSDP_CHUNKS(c, at, left)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = a.residual_scale * float(x[c][i]);
        }
        if (a.y) {
            TX* y = row_of<TX>(a.y, row, a.y_stride);
            FSDP_CHUNKS(c, at, left) store_some(y + at, left, v[c]);
        }
        if (a.h) {
            float s = 0.f;
            FSDP_CHUNKS(c, at, left)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += v[c][i] * v[c][i];
            const float r = rsqrtf(sum(s) / float(hidden) + a.eps);
            TB* h = row_of<TB>(a.h, row, a.h_stride);
            FSDP_CHUNKS(c, at, left) {
                const Eight<TW> w = load_some(static_cast<const TW*>(a.pre) + at, left);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= r * float(w[i]);
                store_some(h + at, left, v[c]);
            }
        }
    }
}

// ------------------------------------------------------------------ gradient

struct NormGradArgs {
    const void *y, *dy, *dh, *branch, *post, *gate, *pre;
    void *dx, *dbranch, *dgate;
    float *part_pre, *part_post, *part_gate;     // [units, hidden], or NULL
    int64_t y_stride, dy_stride, dh_stride, branch_stride, dx_stride, dbranch_stride;
    int64_t tokens, group_rows, unit_rows;
    int64_t units_per_group;                     // > 0: a unit's rows share one row of the gate
    int hidden;
    float eps, residual_scale, branch_scale;
};

// A workgroup takes a unit of consecutive rows and sums the weights' gradients
// over them in registers; the units' sums are joined by join_kernel, in order.
// While a row is worked on the next one is on its way.  A row needs one round of
// sums over the team: with c = branch_scale * gate * post_weight * branch, the
// inner product of c with the gradient of y is that of c with dy, dh * pre_weight
// and y, weighted by row statistics that the same round gives.
template <typename TX, typename TB, typename TW, int kTeam, int kChunks>
__global__ __launch_bounds__(kTeam* kTeams<kTeam>) void norm_grad_kernel(const NormGradArgs a) {
    // 1024 threads have 128 registers each: two chunks leave no room for the next
    // row, the weights and the weights' sums, which then lie in LDS (in registers
    // they spilled: 855 us at 4096 x 16384, which takes 230 so).
    constexpr bool kRoomy = kTeam < 1024 || kChunks == 1;
    constexpr int kGroup = kTeams<kTeam>;
    __shared__ float part[2][6 * (kTeam / 64)];
    __shared__ float joined[kGroup > 1 ? kGroup : 1][kGroup > 1 ? kTeam * kChunks * 8 : 1];
    const int t = threadIdx.x % kTeam, team = threadIdx.x / kTeam;
    const int hidden = a.hidden;
    const int64_t unit = blockIdx.x;
    // Rows by `run`s, one to a team in turn: a row of the gate's tokens where the unit holds whole ones, else one.
    int64_t lo, hi, group = 0, run = 1;
    const bool whole = a.units_per_group == 0;
    if (!whole) {
        group = unit / a.units_per_group;
        lo = group * a.group_rows + unit % a.units_per_group * a.unit_rows;
        hi = min(lo + a.unit_rows, (group + 1) * a.group_rows);
    } else {
        lo = unit * a.unit_rows;
        hi = min(lo + a.unit_rows, a.tokens);
        if (a.gate) {
            run = a.group_rows;
            group = lo / run + team;
        }
    }
    struct Row {
        Eight<TX> y[kChunks], dy[kChunks];
        Eight<TB> dh[kChunks], b[kChunks];
    };
    const auto load = [&](Row& r, int64_t row) {
        FSDP_CHUNKS(c, at, left) {
            if (a.dy) r.dy[c] = load_some(row_of<TX>(a.dy, row, a.dy_stride) + at, left);
            if (a.dh) {
                r.y[c] = load_some(row_of<TX>(a.y, row, a.y_stride) + at, left);
                r.dh[c] = load_some(row_of<TB>(a.dh, row, a.dh_stride) + at, left);
            }
            if (a.branch) r.b[c] = load_some(row_of<TB>(a.branch, row, a.branch_stride) + at, left);
        }
    };
    Eight<TW> wy[kChunks], wb[kChunks];
    Eight<TB> gate[kChunks];
    const auto load_weights = [&](int c, int at, int left) {
        if (a.dh) wy[c] = load_some(static_cast<const TW*>(a.pre) + at, left);
        if (a.post) wb[c] = load_some(static_cast<const TW*>(a.post) + at, left);
    };
    const auto load_gate = [&](int c, int at, int left) {
        if (a.gate) gate[c] = load_some(row_of<TB>(a.gate, group, hidden) + at, left);
    };
    float dpre[kRoomy ? kChunks : 1][8] = {}, dpost[kRoomy ? kChunks : 1][8] = {}, dgate[kChunks][8] = {};
    __shared__ __attribute__((aligned(16))) float wide[2][kRoomy ? 1 : kTeam * kChunks * 8];
    if constexpr (!kRoomy)
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) wide[0][(c * kTeam + t) * 8 + i] = wide[1][(c * kTeam + t) * 8 + i] = 0.f;
    const auto add_wide = [&](int k, int c, const float(&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) wide[k][(c * kTeam + t) * 8 + i] += v[i];
    };
    int64_t row = lo + team * run, in_run = 0;
    Row r, next;
    if constexpr (kRoomy) {
        if (row < hi) {
            load(r, row);
            FSDP_CHUNKS(c, at, left) {
                load_weights(c, at, left);
                load_gate(c, at, left);
            }
        }
    }
    int flip = 0;
    while (row < hi) {
        const bool run_ends = ++in_run == run;
        const int64_t after = row + 1 + (run_ends ? (kGroup - 1) * run : 0);
        if constexpr (kRoomy) {
            if (after < hi) load(next, after);
        } else {
            load(r, row);
        }
        float s[6] = {};             // sums of y^2, dh w y, branch^2, c dy, c dh w, c y
        FSDP_CHUNKS(c, at, left) {
            if constexpr (!kRoomy) {
                load_weights(c, at, left);
                load_gate(c, at, left);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float up = a.dh ? float(r.dh[c][i]) * float(wy[c][i]) : 0.f, y = a.dh ? float(r.y[c][i]) : 0.f;
                s[0] += y * y;
                s[1] += up * y;
                if (a.post) {
                    const float b = float(r.b[c][i]);
                    const float k = b * float(wb[c][i]) * (a.gate ? float(gate[c][i]) : 1.f);
                    s[2] += b * b;
                    if (a.dy) s[3] += k * float(r.dy[c][i]);
                    s[4] += k * up;
                    s[5] += k * y;
                }
            }
        }
        if (a.dh || a.post) {
            group_sum<kTeam, 6>(s, part[flip]);
            flip ^= 1;
        }
        const float per = 1.f / float(hidden);
        // The factors of u = y ry and n = branch rb.  Inverse roots meet what they normalise
        // first: their cubes leave fp32's range for rows beyond 1e12, or (without eps) below 1e-12.
        const float ry = a.dh ? rsqrtf(s[0] * per + a.eps) : 0.f, my = ry * (ry * (s[1] * per));
        const float rb = a.post ? rsqrtf(s[2] * per + a.eps) : 1.f;
        const float mb = a.post ? rb * (rb * (a.branch_scale * (s[3] + ry * s[4] - (ry * s[5]) * my) * per)) : 0.f;
        FSDP_CHUNKS(c, at, left) {
            if constexpr (!kRoomy) {
                load_weights(c, at, left);
                load_gate(c, at, left);
            }
            float g[8], term[8];     // the gradient of y, a row's term of a sum
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[i] = a.dy ? float(r.dy[c][i]) : 0.f;
                if (a.dh) {
                    const float d = float(r.dh[c][i]), u = float(r.y[c][i]) * ry;
                    if constexpr (kRoomy) dpre[c][i] += d * u;
                    else term[i] = d * u;
                    g[i] += d * float(wy[c][i]) * ry - u * my;
                }
            }
            if constexpr (!kRoomy)
                if (a.dh) add_wide(0, c, term);
            if (a.dx) {
                float out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = a.residual_scale * g[i];
                store_some(row_of<TX>(a.dx, row, a.dx_stride) + at, left, out);
            }
            if (a.branch) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float dn = a.branch_scale * g[i];
                    const float b = float(r.b[c][i]), n = b * rb;
                    if (a.gate) {
                        dgate[c][i] += dn * (a.post ? n * float(wb[c][i]) : n);
                        dn *= float(gate[c][i]);
                    }
                    if (a.post) {
                        if constexpr (kRoomy) dpost[c][i] += dn * n;
                        else term[i] = dn * n;
                        dn = rb * (dn * float(wb[c][i])) - n * mb;
                    }
                    g[i] = dn;                   // without post_weight the branch's values do not matter
                }
                if constexpr (!kRoomy)
                    if (a.post) add_wide(1, c, term);
                if (a.dbranch) store_some(row_of<TB>(a.dbranch, row, a.dbranch_stride) + at, left, g);
            }
        }
        if (run_ends) {
            in_run = 0;
            if (a.gate && whole) {
                if (a.dgate) FSDP_CHUNKS(c, at, left) store_some(row_of<TB>(a.dgate, group, hidden) + at, left, dgate[c]);
                FSDP_CHUNKS(c, at, left)
#pragma unroll
                    for (int i = 0; i < 8; ++i) dgate[c][i] = 0.f;
                group += kGroup;
                if constexpr (kRoomy) {
                    if (after < hi) FSDP_CHUNKS(c, at, left) load_gate(c, at, left);
                }
            }
        }
        row = after;
        if constexpr (kRoomy) r = next;
    }
    const auto leave = [&](float* out, const float(&sum)[kChunks][8]) {
        if (!out) return;
        if constexpr (kGroup > 1) {
            __syncthreads();         // `joined` has been read
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) joined[team][(c * kTeam + t) * 8 + i] = sum[c][i];
            __syncthreads();
            for (int j = threadIdx.x; j < hidden; j += kTeam * kGroup) {
                float v = 0.f;
#pragma unroll
                for (int k = 0; k < kGroup; ++k) v += joined[k][j];
                out[unit * hidden + j] = v;
            }
        } else {
            FSDP_CHUNKS(c, at, left) store_some(out + unit * hidden + at, left, sum[c]);
        }
    };
    if constexpr (kRoomy) {
        leave(a.part_pre, dpre);
        leave(a.part_post, dpost);
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float* const out = k == 0 ? a.part_pre : a.part_post;
            float sum[kChunks][8];
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[c][i] = wide[k][(c * kTeam + t) * 8 + i];
            leave(out, sum);
        }
    }
    leave(a.part_gate, dgate);
}

// ------------------------------------------------------------------ host side

constexpr int64_t kMaxGrid = int64_t(1) << 21;   // workgroups of a launch: below 2^31 threads

// f(stream type, block type, weight type) of a call's types.
template <typename F>
fsdp_status with_types(fsdp_dtype stream, fsdp_dtype block, fsdp_dtype weight, F f) {
    const auto inner = [&](auto tb) {
        using TB = decltype(tb);
        if constexpr (std::is_same_v<TB, float>) {
            return f(0.f, 0.f, 0.f);
        } else {
            if (stream == FSDP_DTYPE_F32) return weight == FSDP_DTYPE_F32 ? f(0.f, tb, 0.f) : f(0.f, tb, tb);
            return weight == FSDP_DTYPE_F32 ? f(tb, tb, 0.f) : f(tb, tb, tb);
        }
    };
    return block == FSDP_DTYPE_BF16 ? inner(bf16(0.f)) : block == FSDP_DTYPE_F16 ? inner(f16(0.f)) : inner(0.f);
}

// f(team, chunks) for a row.  kTwo: two chunks a thread in half the threads where
// there is a choice (the forward of 16-bit blocks: 154 instead of 163 us at 8192 x
// 8192, 85 instead of 111 at 8192 x 4097, where the larger team idles by half).
template <bool kTwo, typename F>
fsdp_status with_shape(int64_t hidden, F f) {
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Chunks = std::integral_constant<int, kTwo ? 2 : 1>;
    if (hidden <= 512) return f(std::integral_constant<int, 64>(), One());
    if (hidden <= 1024) return f(std::integral_constant<int, 64>(), Two());
    if (hidden <= 2048) return f(std::integral_constant<int, 256>(), One());
    if (hidden <= 4096) return f(std::integral_constant<int, kTwo ? 256 : 512>(), Chunks());
    if (hidden <= 8192) return f(std::integral_constant<int, kTwo ? 512 : 1024>(), Chunks());
    return f(std::integral_constant<int, 1024>(), Two());
}

// The checks that the norms and their gradient share.
fsdp_status check_norm(int64_t tokens, int64_t hidden, int64_t gate_rows, fsdp_dtype stream, fsdp_dtype block, fsdp_dtype weight,
                       float eps, float residual_scale, float branch_scale, bool branch, bool post, bool gate) {
    if (tokens < 0) return fail(FSDP_ERR_INVALID, "tokens is negative");
    if (hidden < 1) return fail(FSDP_ERR_INVALID, "hidden is below 1");
    if (hidden > FSDP_NORM_MAX_HIDDEN) return fail(FSDP_ERR_OVERFLOW, "hidden is above %d", FSDP_NORM_MAX_HIDDEN);
    if (!known_dtype(stream) || !known_dtype(block) || !known_dtype(weight)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (stream != block && stream != FSDP_DTYPE_F32)
        return fail(FSDP_ERR_INVALID, "the stream must have the block's type or be fp32");
    if (weight != block && weight != FSDP_DTYPE_F32)
        return fail(FSDP_ERR_INVALID, "the weights must have the block's type or be fp32");
    if (!(eps >= 0.f) || !__builtin_isfinite(eps) || !__builtin_isfinite(residual_scale) || !__builtin_isfinite(branch_scale))
        return fail(FSDP_ERR_INVALID, "eps must not be negative, eps and the scales must be finite");
    if (!branch && (post || gate)) return fail(FSDP_ERR_INVALID, "post_weight and gate need a branch");
    if (gate != (gate_rows != 0) || gate_rows < 0) return fail(FSDP_ERR_INVALID, "gate_rows and gate do not agree");
    if (gate && tokens % gate_rows != 0)
        return fail(FSDP_ERR_INVALID, "%lld tokens do not share %lld rows of the gate evenly", (long long)tokens, (long long)gate_rows);
    return FSDP_OK;
}

// How the rows are dealt to units, and where the units' sums lie.
struct GradCut {
    int64_t units = 0, unit_rows = 1, units_per_group = 0;
    int64_t pre = -1, post = -1, gate = -1;      // float offsets in the workspace
    int64_t bytes = 0;
};

// Workgroups per CU: more make more sums to join than they hide (twice as many: 6 %
// slower at 8192 x 4096 and 8192 x 8192, 12 % at 16384 x 1024; half: 6 % slower at
// 8192 x 4096, 16 % at 32768 x 256).  At least four rows to a unit for the same
// reason, but for a few rows, which wait for each other.
int64_t units_wanted(int64_t tokens, int64_t hidden, int cus) {
    const int64_t per_cu = hidden <= 512 ? 4 : hidden <= 4096 ? 2 : 1;
    const int64_t few = std::min(tokens, int64_t(cus) / 2);
    return std::max<int64_t>(1, std::min(int64_t(cus) * per_cu, std::max(few, ceil_div(tokens, 4))));
}

GradCut cut_rows(const fsdp_norm_grad_args& a, int cus) {
    GradCut c;
    if (a.tokens > 0) {
        const int64_t rows = ceil_div(a.tokens, units_wanted(a.tokens, a.hidden, cus));
        const int64_t group = a.gate ? a.tokens / a.gate_rows : 1;
        if (a.gate && group > rows) {
            c.units_per_group = ceil_div(group, rows);
            c.unit_rows = ceil_div(group, c.units_per_group);
            c.units_per_group = ceil_div(group, c.unit_rows);
            c.units = a.gate_rows * c.units_per_group;
        } else {
            c.unit_rows = std::max<int64_t>(1, rows / group) * group;
            c.units = ceil_div(a.tokens, c.unit_rows);
        }
    }
    int64_t at = 0;
    const auto take = [&](bool wanted, int64_t* where) {
        if (!wanted) return;
        *where = at;
        at += round_up(c.units * a.hidden, 64);
    };
    take(a.dpre_weight, &c.pre);
    take(a.dpost_weight, &c.post);
    take(a.dgate && c.units_per_group > 0, &c.gate);
    c.bytes = at * 4;
    return c;
}

fsdp_status check_grad(const fsdp_norm_grad_args& a) {
    fsdp_status st = check_norm(a.tokens, a.hidden, a.gate_rows, a.stream_dtype, a.block_dtype, a.weight_dtype, a.eps,
                                a.residual_scale, a.branch_scale, a.branch, a.post_weight, a.gate);
    if (st != FSDP_OK) return st;
    if (!a.dh != !a.pre_weight && a.tokens > 0) return fail(FSDP_ERR_INVALID, "dh and pre_weight go together");
    if (a.dbranch && !a.branch && a.tokens > 0) return fail(FSDP_ERR_INVALID, "dbranch needs a branch");
    if (a.dpre_weight && !a.pre_weight) return fail(FSDP_ERR_INVALID, "dpre_weight needs pre_weight");
    if (a.dpost_weight && !a.post_weight) return fail(FSDP_ERR_INVALID, "dpost_weight needs post_weight");
    if (a.dgate && !a.gate) return fail(FSDP_ERR_INVALID, "dgate needs a gate");
    // The rows that a launch joins into dgate: with tokens, fewer than the units of the largest device.
    if (a.tokens == 0 && a.gate_rows > 60000) return fail(FSDP_ERR_OVERFLOW, "too many rows of the gate without tokens");
    Checked m;
    const int64_t t = a.tokens, h = a.hidden;
    m.add_in_place("y", a.y, t, h, a.y_stride, a.stream_dtype, a.dh);
    m.add_in_place("dy", a.dy, t, h, a.dy_stride, a.stream_dtype, false);
    m.add_in_place("dh", a.dh, t, h, a.dh_stride, a.block_dtype, false);
    m.add_in_place("branch", a.branch, t, h, a.branch_stride, a.block_dtype, false);
    m.add_vector("post_weight", a.post_weight, h, a.weight_dtype, false);
    m.add("gate", a.gate, a.gate_rows, h, h, a.block_dtype, false);
    m.add_vector("pre_weight", a.pre_weight, h, a.weight_dtype, false);
    m.add("dx", a.dx, t, h, a.dx_stride, a.stream_dtype, false, true, a.dy);
    m.add("dbranch", a.dbranch, t, h, a.dbranch_stride, a.block_dtype, false, true, a.branch, a.dh);
    m.add_vector("dpre_weight", a.dpre_weight, h, a.weight_dtype, false, true);
    m.add_vector("dpost_weight", a.dpost_weight, h, a.weight_dtype, false, true);
    m.add("dgate", a.dgate, a.gate_rows, h, h, a.block_dtype, false, true);
    return m.done();
}

}  // namespace
}  // namespace fsdp_block

using namespace fsdp_block;

extern "C" fsdp_status fsdp_block_norm(const fsdp_norm_args* args, hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_norm_args& a = *args;
    fsdp_status st = check_norm(a.tokens, a.hidden, a.gate_rows, a.stream_dtype, a.block_dtype, a.weight_dtype, a.eps,
                                a.residual_scale, a.branch_scale, a.branch, a.post_weight, a.gate);
    if (st != FSDP_OK) return st;
    if (a.tokens > 0 && !a.y && !a.h) return fail(FSDP_ERR_INVALID, "neither y nor h is wanted");
    if (a.tokens > 0 && a.h && !a.pre_weight) return fail(FSDP_ERR_INVALID, "h needs pre_weight");
    Checked m;
    m.add_in_place("x", a.x, a.tokens, a.hidden, a.x_stride, a.stream_dtype, true);
    m.add_in_place("branch", a.branch, a.tokens, a.hidden, a.branch_stride, a.block_dtype, false);
    m.add_vector("post_weight", a.post_weight, a.hidden, a.weight_dtype, false);
    m.add("gate", a.gate, a.gate_rows, a.hidden, a.hidden, a.block_dtype, false);
    m.add_vector("pre_weight", a.pre_weight, a.hidden, a.weight_dtype, false);
    m.add("y", a.y, a.tokens, a.hidden, a.y_stride, a.stream_dtype, false, true, a.x);
    m.add("h", a.h, a.tokens, a.hidden, a.h_stride, a.block_dtype, false, true, a.branch);
    if ((st = m.done()) != FSDP_OK || a.tokens == 0) return st;
    const NormArgs k{a.x, a.branch, a.post_weight, a.gate, a.pre_weight, a.y, a.h, a.x_stride, a.branch_stride, a.y_stride,
                     a.h_stride, a.tokens, a.gate ? a.tokens / a.gate_rows : a.tokens, int(a.hidden), a.eps,
                     a.residual_scale, a.branch_scale};
    return with_types(a.stream_dtype, a.block_dtype, a.weight_dtype, [&](auto tx, auto tb, auto tw) {
        return with_shape<!std::is_same_v<decltype(tb), float>>(a.hidden, [&](auto team, auto chunks) {
            constexpr int kTeam = decltype(team)::value;
            const int64_t grid = std::min(kMaxGrid, ceil_div(a.tokens, kTeams<kTeam>));
            return launch(norm_kernel<decltype(tx), decltype(tb), decltype(tw), kTeam, decltype(chunks)::value>, k,
                          dim3(unsigned(grid)), kTeam * kTeams<kTeam>, stream);
        });
    });
}

extern "C" fsdp_status fsdp_block_norm_grad_workspace(const fsdp_norm_grad_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    fsdp_status st = check_grad(*args);
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    *bytes = cut_rows(*args, cus).bytes;
    return FSDP_OK;
}

extern "C" fsdp_status fsdp_block_norm_grad(const fsdp_norm_grad_args* args, void* workspace, int64_t workspace_bytes,
                                            hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_norm_grad_args& a = *args;
    fsdp_status st = check_grad(a);
    if (st != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    const GradCut cut = cut_rows(a, cus);
    if ((st = check_workspace(workspace, workspace_bytes, cut.bytes)) != FSDP_OK) return st;
    float* const ws = static_cast<float*>(workspace);
    const auto at = [&](int64_t offset) { return offset < 0 ? nullptr : ws + offset; };
    if (a.tokens > 0) {
        const NormGradArgs k{a.y, a.dy, a.dh, a.branch, a.post_weight, a.gate, a.pre_weight, a.dx, a.dbranch, a.dgate,
                             at(cut.pre), at(cut.post), at(cut.gate), a.y_stride, a.dy_stride, a.dh_stride,
                             a.branch_stride, a.dx_stride, a.dbranch_stride, a.tokens,
                             a.gate ? a.tokens / a.gate_rows : a.tokens, cut.unit_rows, cut.units_per_group,
                             int(a.hidden), a.eps, a.residual_scale, a.branch_scale};
        st = with_types(a.stream_dtype, a.block_dtype, a.weight_dtype, [&](auto tx, auto tb, auto tw) {
            return with_shape<false>(a.hidden, [&](auto team, auto chunks) {
                constexpr int kTeam = decltype(team)::value;
                return launch(norm_grad_kernel<decltype(tx), decltype(tb), decltype(tw), kTeam, decltype(chunks)::value>, k,
                              dim3(unsigned(cut.units)), kTeam * kTeams<kTeam>, stream);
            });
        });
        if (st != FSDP_OK) return st;
    }
    Join j(int(a.hidden));
    j.add(a.dpre_weight, at(cut.pre), cut.units, 1, a.weight_dtype);
    j.add(a.dpost_weight, at(cut.post), cut.units, 1, a.weight_dtype);
    // Without tokens no unit has written the gate's gradient: it is joined from none.
    if (a.tokens == 0 || cut.units_per_group > 0)
        j.add(a.dgate, at(cut.gate), cut.units_per_group, a.gate_rows, a.block_dtype);
    return j.run(a.block_dtype, stream);
}
