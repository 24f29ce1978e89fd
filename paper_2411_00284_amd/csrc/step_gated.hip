// A gated feed-forward's two projections with their activation and product, its
// gradient, and a linear layer's gradient from an input and a pre-activation in 8
// bits (include/fsdp_step.h).
//
// The products take the tiles of block_product.h. Forward, a tile holds the same
// columns of both projections, so that the activation and the product of the two are
// made in its epilogue and x is read once for both. Backward, one pass makes dg and du
// side by side in a row of the workspace; dx is then one product whose sum runs over
// both weights, and the weights' gradients are one product of twice the rows.

#include "block_cut.h"
#include "block_join.h"
#include "block_lay.h"
#include "step_product.h"

#include <algorithm>

namespace fsdp_block {
namespace {

// ------------------------------------------------------------------ few rows

// As many rows of each weight to a wave as keep eight loads in flight.
template <int kRows>
constexpr int kGatedOut = kRows > 2 ? 2 : 1;

// g and u of at most kRows rows of x: a wave takes kGatedOut rows of both weights,
// which are read once, past the caches. kTogetherK: the four waves of a workgroup take the same
// rows, every fourth part of k each, where there are too few rows to fill the card otherwise
// (2 x 104 with k = 20401 in fp16: 7.6 us instead of 24.6).
//
// Bound by HBM: 1 x 14336 x 4096 in bf16 takes 35.6 us, 6.6 TB/s of both weights.
template <typename T, int kRows, bool kTogetherK>
__global__ __launch_bounds__(256) void gated_row_kernel(const PairProduct p) {
    constexpr int kOut = kGatedOut<kRows>, kTogether = 4 / kOut;
    __shared__ float sums[4][2][kOut][kRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j0 = (kTogetherK ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + wave) * kOut;
    if (j0 >= p.inner) return;                   // not in part: with kTogetherK the whole workgroup or none
    const T* w[2][kOut];
#pragma unroll
    for (int o = 0; o < kOut; ++o) {
        const int64_t row = min(j0 + o, p.inner - 1);
        w[0][o] = static_cast<const T*>(p.b) + row * p.b_stride;
        w[1][o] = static_cast<const T*>(p.b2) + row * p.b2_stride;
    }
    const T* x = static_cast<const T*>(p.a);
    float sum[2][kOut][kRows] = {};
    const auto add = [&](int64_t k, int n) {
        Eight<T> v[2][kOut];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int o = 0; o < kOut; ++o) v[h][o] = n == 8 && sizeof(T) == 2 ? load8_once(w[h][o] + k) : load_some(w[h][o] + k, n);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const Eight<T> u = load_some(x + min(int64_t(i), p.m - 1) * p.a_stride + k, n);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int o = 0; o < kOut; ++o)
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[h][o][i] += float(v[h][o][c]) * float(u[c]);
        }
    };
    constexpr int64_t kStep = kTogetherK ? 2048 : 512;
    int64_t k = (kTogetherK ? threadIdx.x : lane) * 8;
#pragma unroll kTogether
    for (; k + 8 <= p.k; k += kStep) add(k, 8);
    if (k < p.k) add(k, int(p.k - k));
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
            for (int i = 0; i < kRows; ++i) sum[h][o][i] = wave_sum(sum[h][o][i]);
    if constexpr (kTogetherK) {
        if (lane == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int o = 0; o < kOut; ++o)
#pragma unroll
                    for (int i = 0; i < kRows; ++i) sums[wave][h][o][i] = sum[h][o][i];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int o = 0; o < kOut; ++o)
#pragma unroll
                for (int i = 0; i < kRows; ++i)
                    sum[h][o][i] = (sums[0][h][o][i] + sums[1][h][o][i]) + (sums[2][h][o][i] + sums[3][h][o][i]);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (lane == i && lane < p.m)
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                const int64_t j = j0 + o;
                if (j >= p.inner) continue;
                const float g = sum[0][o][i], u = sum[1][o][i];
                static_cast<T*>(p.e.out)[i * p.e.out_stride + j] = T(act_value<sizeof(T) == 4>(g, p.e.act) * u);
                if (p.gate) static_cast<T*>(p.gate)[i * p.gate_stride + j] = T(g);
                if (p.up) static_cast<T*>(p.up)[i * p.up_stride + j] = T(u);
            }
}

// ------------------------------------------------------------------ dg, du and dz

// A row's eight columns of what is kept, in the type or in 8 bits.
template <typename T, bool kSaved>
struct Kept {
    Eight<T> v;
    i8x8 codes;
    float scale;
    __device__ __forceinline__ void load(const void* p, const uint8_t* scales, int64_t stride, int64_t scales_stride, int64_t i, int64_t j,
                                         int left) {
        if constexpr (kSaved) {
            const int8_t* const at = static_cast<const int8_t*>(p) + i * stride + j;
            codes = left >= 8 ? load_codes_once(at) : load_codes(at, left);
            scale = scale_value(scales[i * scales_stride + j / FSDP_STEP_GROUP]);
        } else {
            const T* const at = static_cast<const T*>(p) + i * stride + j;
            v = left >= 8 && sizeof(T) == 2 ? load8_once(at) : load_some(at, left);
        }
    }
    __device__ __forceinline__ float operator[](int c) const {
        if constexpr (kSaved) return float(codes[c]) * scale;
        else return float(v[c]);
    }
};

struct GatedSlopeArgs {
    const void *dout, *gate, *up;
    const uint8_t *gate_scales, *up_scales;
    void *dz, *out;                  // dz or NULL
    int64_t dout_stride, gate_stride, up_stride, gate_scales_stride, up_scales_stride, dz_stride, out_stride;
    int64_t m, n, split, part_rows;
    int act;
};

// A workgroup takes 512 columns of part_rows rows, a row per wave at a time. dg lies
// in columns 0 .. of dz, du from `split` on, zeros after each up to whole lines.
//
// dg and du are rounded to the type here: the matrix instructions take factors of 16 bits.
//
// Bound by HBM: 4096 x 14336 in bf16 from projections in 8 bits, SiLU, moves 590 MB in 98 us, 6.0 TB/s.
template <typename T, bool kSaved>
__global__ __launch_bounds__(256) void gated_slope_kernel(const GatedSlopeArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = int64_t(blockIdx.x) * 512 + lane * 8;
    const int left = int(min(a.n - j, int64_t(8)));
    if (j >= a.split) return;
    const int64_t hi = min((int64_t(blockIdx.y) + 1) * a.part_rows, a.m);
    for (int64_t i = int64_t(blockIdx.y) * a.part_rows + wave; i < hi; i += 4) {
        float dg[8] = {}, du[8] = {}, out[8];
        if (left > 0) {
            Kept<T, kSaved> g, u;
            Kept<T, false> d;
            d.load(a.dout, nullptr, a.dout_stride, 0, i, j, left);
            g.load(a.gate, a.gate_scales, a.gate_stride, a.gate_scales_stride, i, j, left);
            u.load(a.up, a.up_scales, a.up_stride, a.up_scales_stride, i, j, left);
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    float value, slope;
                    act_both<sizeof(T) == 4>(g[c], decltype(act)::value, value, slope);
                    out[c] = value * u[c];
                    const bool held = c < left;          // past the row's end the values stand for nothing
                    dg[c] = held ? d[c] * u[c] * slope : 0.f;
                    du[c] = held ? d[c] * value : 0.f;
                }
            });
            if (a.out) store_some(static_cast<T*>(a.out) + i * a.out_stride + j, left, out);
        }
        if (a.dz) {
            T* const dz = static_cast<T*>(a.dz) + i * a.dz_stride + j;
            store_some(dz, 8, dg);
            store_some(dz + a.split, 8, du);
        }
    }
}

struct SavedSlopeArgs {
    const void *dout, *pre, *times;
    const uint8_t* pre_scales;
    void *dz, *dtimes;               // dz or NULL
    float* part;                     // [row parts, n] sums of dz, or NULL
    int64_t dout_stride, pre_stride, pre_scales_stride, times_stride, dz_stride, dtimes_stride;
    int64_t m, n, wide, part_rows;   // dz has `wide` columns, zeros from n on
    int act;
};

// As gated_slope_kernel, for a linear layer: dz = dout * times * act'(z), and its sums
// over the rows.
//
// 2048 x 14336 in fp16 from 8 bits with GELU takes 45 us: the vector units are busy 98 % of it.
template <typename T, bool kSaved>
__global__ __launch_bounds__(256) void saved_slope_kernel(const SavedSlopeArgs a) {
    __shared__ float sums[4][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = int64_t(blockIdx.x) * 512 + lane * 8;
    const int left = int(min(a.n - j, int64_t(8)));
    const int64_t hi = min((int64_t(blockIdx.y) + 1) * a.part_rows, a.m);
    float sum[8] = {};
    if (j < a.wide)
        for (int64_t i = int64_t(blockIdx.y) * a.part_rows + wave; i < hi; i += 4) {
            float dz[8] = {}, df[8];
            if (left > 0) {
                Kept<T, false> d, f;
                Kept<T, kSaved> z;
                d.load(a.dout, nullptr, a.dout_stride, 0, i, j, left);
                if (a.pre) z.load(a.pre, a.pre_scales, a.pre_stride, a.pre_scales_stride, i, j, left);
                if (a.times) f.load(a.times, nullptr, a.times_stride, 0, i, j, left);
                with_act(a.act, [&](auto act) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        float value = 1.f, slope = 1.f, v = d[c];
                        if (a.pre) act_both<sizeof(T) == 4>(z[c], decltype(act)::value, value, slope);
                        df[c] = v * value;
                        if (a.times) v *= f[c];
                        if (decltype(act)::value != FSDP_ACT_NONE) v *= slope;
                        dz[c] = c < left ? v : 0.f;
                        sum[c] += dz[c];
                    }
                });
                if (a.dtimes) store_some(static_cast<T*>(a.dtimes) + i * a.dtimes_stride + j, left, df);
            }
            if (a.dz) store_some(static_cast<T*>(a.dz) + i * a.dz_stride + j, 8, dz);
        }
    if (!a.part) return;
#pragma unroll
    for (int c = 0; c < 8; ++c) sums[wave][lane * 8 + c] = sum[c];
    __syncthreads();
    for (int c = threadIdx.x; c < 512; c += 256) {
        const int64_t column = int64_t(blockIdx.x) * 512 + c;
        if (column < a.n) a.part[blockIdx.y * a.n + column] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    }
}

// ------------------------------------------------------------------ host side: products

int64_t row_stride(int64_t rows, int64_t cols, int64_t stride) { return rows > 1 ? stride : round_up(cols, 8); }

// The forms of a product, as block_cut.h has them: in 16 bits those of step_tile.h (`steps` is
// their ring), then block_product.h's; a forward product has none of 64 x 64. Times from a round of
// 256 workgroups (or 512 of two on a CU) at k = 2560 and 10240, the three kinds of product within
// 5 % of each other. (Tiles of 128 x 256 take 0.83 to 0.93 us a step, two of 128 x 128 on a CU
// the same: they are not built.)
constexpr Form kRings[] = {
    {256, 256, 5, 1, 1.25, 1.45, 7.0},
    {128, 128, 5, 2, 0.50, 0.92, 5.0},
    {128, 128, 10, 1, 0.42, 0.45, 4.5},
    {64, 128, 4, 1, 0.28, 0.32, 4.0},
    {64, 64, 8, 1, 0.16, 0.21, 4.0},
};
// fp32, from products of 2048 x 1024 x 688 to 5000 x 2500 x 1500. A gradient's small tiles are those
// of 64 x 64, two on a CU: the weights' gradients of 2048 x 688 -> 1024 take 67 us instead of 74 in
// tiles of 64 x 128, of 59 x 28672 -> 256 the whole call 114 instead of 164. A linear layer's gradient
// has the forms and the parts of k that it has without 8 bits: where no part is longer than a run
// (step_product.h), 512 k, its bits too. Longer ones are summed in runs here and one term after the other
// there: 4096 x 1024 -> 4096 is 4.1e-7 off 64 bits (2-norm) from an x in 8 bits, in 561 us, and 1.14e-6
// from its values, in 497.
constexpr Form kForwards32[] = {{128, 128, 2, 2, 2.10, 4.15, 5.0}, {64, 128, 4, 1, 1.22, 1.28, 4.0}};
constexpr Form kGrads32[] = {{128, 128, 2, 2, 2.10, 4.15, 5.0}, {64, 64, 4, 2, 0.58, 1.14, 3.5}};
constexpr Forms kForward16{kRings, 4, kRings + 1, 1}, kGrad16{kRings, 5, kRings + 1, 1};
constexpr Forms kForward32{kForwards32, 2, nullptr, 0}, kGrad32{kGrads32, 2, nullptr, 0};
const Forms& forward_forms(fsdp_dtype dtype) { return dtype == FSDP_DTYPE_F32 ? kForward32 : kForward16; }
const Forms& grad_forms(fsdp_dtype dtype, bool two) { return dtype != FSDP_DTYPE_F32 ? kGrad16 : two ? kGrad32 : kLinear32; }

// A product's launches: `p` has its operands and epilogue, `c` says how.
template <typename Kind>
fsdp_status launch_pair(const PairProduct& p, const Form& f, fsdp_dtype dtype, hipStream_t stream) {
    constexpr bool kSmallest = !std::is_same<Kind, GatedForward>::value;
    const dim3 grid(unsigned(ceil_div(p.m - p.first_i, f.tile_m) * ceil_div(p.n - p.first_j, f.tile_n) * p.count));
    if (dtype == FSDP_DTYPE_F32) {
        if (f.tile_m == 128) return launch(pair_kernel<float, Kind, 128, 128, 2>, p, grid, 256, stream);
        if constexpr (kSmallest)
            if (f.tile_n == 64) return launch(pair_kernel<float, Kind, 64, 64, 4>, p, grid, 256, stream);
        return launch(pair_kernel<float, Kind, 64, 128, 4>, p, grid, 256, stream);
    }
    const auto of = [&](auto type) {
        using T = decltype(type);
        if (f.tile_m == 256) return launch(ring_kernel<T, Kind, 256, 5>, p, grid, 256, stream);
        if constexpr (kSmallest)
            if (f.tile_n == 64) return launch(pair_kernel<T, Kind, 64, 64, 8>, p, grid, 256, stream);
        if (f.tile_m == 64) return launch(pair_kernel<T, Kind, 64, 128, 4>, p, grid, 256, stream);
        return f.steps == 5 ? launch(ring_kernel<T, Kind, 128, 5>, p, grid, 256, stream)
                            : launch(ring_kernel<T, Kind, 128, 10>, p, grid, 256, stream);
    };
    return dtype == FSDP_DTYPE_BF16 ? of(bf16(0.f)) : of(f16(0.f));
}

template <typename Kind>
fsdp_status run_pair(PairProduct p, const Cut& c, fsdp_dtype dtype, char* ws, hipStream_t stream) {
    if (p.m == 0 || p.n == 0) return FSDP_OK;
    p.part_k = c.part_k;
    p.count = c.count;
    p.parts = c.parts < 0 ? nullptr : reinterpret_cast<float*>(ws + c.parts);
    fsdp_status st;
    if (c.rest) {
        const int64_t m = p.m, n = p.n, inner = p.inner;
        constexpr bool kForward = std::is_same<Kind, GatedForward>::value;
        if (c.rest_rows) p.m = c.rest_at;
        else p.n = c.rest_at;
        if (kForward) p.inner = p.n / 2;
        if ((st = launch_pair<Kind>(p, *c.form, dtype, stream)) != FSDP_OK) return st;
        p.m = m;
        p.n = n;
        p.inner = inner;
        (c.rest_rows ? p.first_i : p.first_j) = c.rest_at;
        return launch_pair<Kind>(p, *c.rest, dtype, stream);
    }
    if ((st = launch_pair<Kind>(p, *c.form, dtype, stream)) != FSDP_OK || c.count == 1) return st;
    const dim3 grid(unsigned(std::min<int64_t>(ceil_div(p.m * ceil_div(p.n, 8), 256), 1 << 13)));
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if constexpr (std::is_same<Kind, GatedForward>::value) return launch(join_gated_kernel<T>, p, grid, 256, stream);
        else return launch(join_pair_kernel<T, Kind>, p, grid, 256, stream);
    });
}

// Offsets in the workspace.
struct Room {
    int64_t bytes = 0;
    int64_t take(int64_t n) {
        const int64_t at = bytes;
        bytes += round_up(n, 256);
        return at;
    }
    int64_t laid(const Source& o, fsdp_dtype dtype) { return take(o.rows * lined(o.cols, dtype) * elem_bytes(dtype)); }
};

void add_parts(Cut& c, const Shape& s, int64_t columns, Room& room) {
    if (c.count > 1) c.parts = room.take(int64_t(c.count) * s.m * columns * 4);
}

// As check_sizes of the linear layer: what launches and 32-bit row counts hold.
fsdp_status check_sizes(int64_t m, int64_t n, int64_t both, int64_t k, fsdp_dtype dtype, fsdp_activation act) {
    if (m < 0 || n < 0 || k < 1) return fail(FSDP_ERR_INVALID, "m and n must not be negative, k must be at least 1");
    if (!known_dtype(dtype)) return fail(FSDP_ERR_INVALID, "unknown dtype");
    if (act < FSDP_ACT_NONE || act > FSDP_ACT_GELU_TANH) return fail(FSDP_ERR_INVALID, "unknown activation");
    const int64_t size = INT32_MAX / 2 / both;
    if (m > size || n > size || k > size) return fail(FSDP_ERR_OVERFLOW, "a size is 2^%d or more", both == 2 ? 29 : 30);
    // Of dz with each part in whole lines.
    const int64_t most = int64_t(1) << 22, wide = both * ceil_div(n, 64);
    if (ceil_div(m, 64) * wide > most || ceil_div(m, 64) * ceil_div(k, 64) > most || wide * ceil_div(k, 64) > most)
        return fail(FSDP_ERR_OVERFLOW, "a product has too many tiles");
    return FSDP_OK;
}

// ------------------------------------------------------------------ host side: forward

// A matrix that may be in 8 bits: values, or codes and scales.
void add_kept(Checked& c, const char* name, const char* scales_name, const void* p, const void* scales, int64_t rows, int64_t cols,
              int64_t stride, int64_t scales_stride, fsdp_dtype dtype, bool needed, bool output) {
    c.add(name, p, rows, cols, stride, scales ? kBytes : dtype, needed, output);
    c.add(scales_name, scales, rows, ceil_div(cols, FSDP_STEP_GROUP), scales_stride, kBytes, false, output);
}

fsdp_status check_gated(const fsdp_step_gated_args& a) {
    const fsdp_status st = check_sizes(a.m, a.n, 2, a.k, a.dtype, a.activation);
    if (st != FSDP_OK) return st;
    const bool any = a.m > 0 && a.n > 0;
    if (any && !a.gate != !a.up) return fail(FSDP_ERR_INVALID, "gate and up go together");
    if (any && !a.gate_scales != !a.up_scales) return fail(FSDP_ERR_INVALID, "gate_scales and up_scales go together");
    if (any && a.gate_scales && !a.gate) return fail(FSDP_ERR_INVALID, "gate_scales needs gate");
    Checked c;
    c.add("x", a.x, a.m, a.k, a.x_stride, a.dtype, a.n > 0);
    c.add("gate_weight", a.gate_weight, a.n, a.k, a.gate_weight_stride, a.dtype, a.m > 0);
    c.add("up_weight", a.up_weight, a.n, a.k, a.up_weight_stride, a.dtype, a.m > 0);
    add_kept(c, "gate", "gate_scales", a.gate, a.gate_scales, a.m, a.n, a.gate_stride, a.gate_scales_stride, a.dtype, false, true);
    add_kept(c, "up", "up_scales", a.up, a.up_scales, a.m, a.n, a.up_stride, a.up_scales_stride, a.dtype, false, true);
    c.add("out", a.out, a.m, a.n, a.out_stride, a.dtype, true, true);
    return c.done();
}

struct Forward {
    Source x, gate, up;
    Shape shape;
    Cut cut;
    int64_t pad[3] = {-1, -1, -1};
    int64_t bytes = 0;
    int cus = 0;
};

// Up to four rows go without tiles, unless 32 columns have to be seen together.
bool by_rows(const fsdp_step_gated_args& a, const Shape& s) { return row_form(s) && !a.gate_scales; }

Forward forward_of(const fsdp_step_gated_args& a) {
    Forward f;
    f.x = {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false};
    f.gate = {a.gate_weight, a.n, a.k, row_stride(a.n, a.k, a.gate_weight_stride), false};
    f.up = {a.up_weight, a.n, a.k, row_stride(a.n, a.k, a.up_weight_stride), false};
    f.shape = {a.m, 2 * a.n, a.k, a.dtype, false, false, laid_stride(f.x, a.dtype),
               std::max(laid_stride(f.gate, a.dtype), laid_stride(f.up, a.dtype))};
    return f;
}

fsdp_status check_reach(const fsdp_step_gated_args& a, const Forward& f) {
    return by_rows(a, f.shape) ? FSDP_OK : check_reach(f.shape, forward_forms(a.dtype), false);
}

void plan_forward(const fsdp_step_gated_args& a, int cus, Forward& f) {
    Room room;
    if (a.m > 0 && a.n > 0 && !by_rows(a, f.shape)) {
        f.cut = choose(f.shape, cus, forward_forms(a.dtype), false);
        const Source* const from[3] = {&f.x, &f.gate, &f.up};
        for (int w = 0; w < 3; ++w)
            if (!on_grid(*from[w], a.dtype)) f.pad[w] = room.laid(*from[w], a.dtype);
        add_parts(f.cut, f.shape, 2 * part_columns(a.n), room);
    }
    f.bytes = room.bytes;
}

fsdp_status ready_forward(const fsdp_step_gated_args& a, Forward& f) {
    fsdp_status st = check_gated(a);
    if (st != FSDP_OK) return st;
    f = forward_of(a);
    if ((st = check_reach(a, f)) != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    f.cus = cus;
    plan_forward(a, cus, f);
    return FSDP_OK;
}

// ------------------------------------------------------------------ host side: gradients

// What both gradients are to the products: dz of one part or two.
struct Grad {
    int64_t m = 0, n = 0, k = 0, split = 0, wide = 0;    // dz has `wide` columns
    fsdp_dtype dtype = 0;
    int act = 0;
    bool two = false, dx = false, dweight = false, saved_x = false;
    bool as_is = false;              // dz is dout itself
    Source weight[2] = {}, x = {}, dout = {};
    Shape dx_shape, dw_shape;
    Cut dx_cut, dw_cut;
    int64_t part_rows = 1, row_parts = 0;
    int64_t dz = -1, sums = -1, restored = -1, pad[2] = {-1, -1}, pad_x = -1, bytes = 0;
};

// Whether the two weights are read where they lie: dx's product steps from one to the
// other with one stride.
bool joined(const Grad& g) {
    const bool first = on_grid(g.weight[0], g.dtype);
    return !g.two ? first : first && on_grid(g.weight[1], g.dtype) && g.weight[0].stride == g.weight[1].stride;
}

void shape_grad(Grad& g) {
    g.split = lined(g.n, g.dtype);
    g.wide = g.two ? 2 * g.split : g.as_is ? g.n : g.split;
    const int64_t dz_stride = g.as_is ? laid_stride(g.dout, g.dtype) : g.wide;
    const int64_t weight_stride = joined(g) ? g.weight[0].stride : lined(g.k, g.dtype);
    const int64_t x_stride = g.saved_x ? lined(g.k, g.dtype) : laid_stride(g.x, g.dtype);
    g.dx_shape = {g.m, g.k, g.wide, g.dtype, false, true, dz_stride, weight_stride};
    g.dw_shape = {g.two ? g.split + g.n : g.n, g.k, g.m, g.dtype, true, true, dz_stride, x_stride};
}

fsdp_status check_reach(const Grad& g) {
    fsdp_status st = FSDP_OK;
    if (g.dx && g.n > 0) st = check_reach(g.dx_shape, grad_forms(g.dtype, g.two));
    return st == FSDP_OK && g.dweight ? check_reach(g.dw_shape, grad_forms(g.dtype, g.two)) : st;
}

void plan_grad(Grad& g, int cus, bool dz, bool sums) {
    Room room;
    if (g.m > 0 && g.n > 0) {
        const int64_t columns = ceil_div(g.split, 512);
        g.part_rows = std::max<int64_t>(4, round_up(ceil_div(g.m * columns, 8 * int64_t(cus)), 4));
        g.row_parts = ceil_div(g.m, g.part_rows);
        if (dz && g.as_is) {
            if (!on_grid(g.dout, g.dtype)) g.dz = room.laid(g.dout, g.dtype);
        } else if (dz) {
            g.dz = room.take(g.m * g.wide * elem_bytes(g.dtype));
        }
        if (sums) g.sums = room.take(g.row_parts * g.n * 4);
        if (g.dweight && g.saved_x) g.restored = room.take(g.m * lined(g.k, g.dtype) * elem_bytes(g.dtype));
        else if (g.dweight && !on_grid(g.x, g.dtype)) g.pad_x = room.laid(g.x, g.dtype);
    }
    // The two products follow each other on the stream: they share what each needs.
    Room first = room, second = room;
    if (g.dx) {
        g.dx_cut = choose(g.dx_shape, cus, grad_forms(g.dtype, g.two));
        if (g.m > 0 && g.n > 0) {
            if (!joined(g))
                for (int w = 0; w < (g.two ? 2 : 1); ++w) g.pad[w] = first.laid(g.weight[w], g.dtype);
            add_parts(g.dx_cut, g.dx_shape, round_up(g.k, 8), first);
        }
    }
    if (g.dweight) {
        g.dw_cut = choose(g.dw_shape, cus, grad_forms(g.dtype, g.two));
        if (g.m > 0 && g.n > 0) add_parts(g.dw_cut, g.dw_shape, round_up(g.k, 8), second);
    }
    g.bytes = std::max(first.bytes, second.bytes);
}

// dx and the weights' gradients from dz in the workspace.
fsdp_status run_products(const Grad& g, const void* codes, const void* scales, int64_t scales_stride, void* dx, int64_t dx_stride,
                         void* dweight, int64_t dweight_stride, void* dweight2, int64_t dweight2_stride, char* ws, hipStream_t stream) {
    fsdp_status st = FSDP_OK;
    PairProduct p{};
    p.a = g.dz >= 0 ? ws + g.dz : g.dout.p;
    p.a_stride = g.dx_shape.stride_a;
    p.inner = g.n;
    p.split = g.two ? g.split : INT64_MAX / 2;
    if (g.as_is && g.dz >= 0) {
        Pads<2> pads;
        pads.add(g.dout, g.dtype, ws + g.dz);
        if ((st = pads.run(stream)) != FSDP_OK) return st;
    }
    if (dx) {
        Pads<2> pads;
        const void* from[2] = {g.weight[0].p, g.weight[1].p};
        p.b_stride = g.dx_shape.stride_b;
        for (int w = 0; w < 2; ++w)
            if (g.pad[w] >= 0) {
                pads.add(g.weight[w], g.dtype, ws + g.pad[w]);
                from[w] = ws + g.pad[w];
            }
        if ((st = pads.run(stream)) != FSDP_OK) return st;
        p.b = from[0];
        p.b2 = from[1];
        p.b2_stride = p.b_stride;
        p.m = g.m;
        p.n = g.k;
        p.k = g.n > 0 ? g.wide : 0;
        p.e.out = dx;
        p.e.out_stride = dx_stride;
        if ((st = run_pair<PairInput>(p, g.dx_cut, g.dtype, ws, stream)) != FSDP_OK) return st;
    }
    if (!dweight) return st;
    p.b = g.x.p;
    p.b_stride = g.dw_shape.stride_b;
    if (g.restored >= 0) {
        p.b = ws + g.restored;
        st = restore(codes, g.x.stride, scales, scales_stride, ws + g.restored, p.b_stride, g.m, g.k, p.b_stride, g.dtype, stream);
        if (st != FSDP_OK) return st;
    } else if (g.pad_x >= 0) {
        Pads<2> pads;
        pads.add(g.x, g.dtype, ws + g.pad_x);
        if ((st = pads.run(stream)) != FSDP_OK) return st;
        p.b = ws + g.pad_x;
    }
    p.m = g.dw_shape.m;
    p.n = g.k;
    p.k = g.m;
    p.e.out = dweight;
    p.e.out_stride = dweight_stride;
    p.out2 = dweight2;
    p.out2_stride = dweight2_stride;
    return run_pair<PairWeights>(p, g.dw_cut, g.dtype, ws, stream);
}

fsdp_status check_gated_grad(const fsdp_step_gated_grad_args& a) {
    const fsdp_status st = check_sizes(a.m, a.n, 2, a.k, a.dtype, a.activation);
    if (st != FSDP_OK) return st;
    const bool any = a.dx || a.dgate_weight || a.out;
    if (a.n > 0 && !a.dgate_weight != !a.dup_weight) return fail(FSDP_ERR_INVALID, "dgate_weight and dup_weight go together");
    if (a.m > 0 && a.n > 0 && !a.gate_scales != !a.up_scales) return fail(FSDP_ERR_INVALID, "gate_scales and up_scales go together");
    Checked c;
    c.add_in_place("dout", a.dout, a.m, a.n, a.dout_stride, a.dtype, any);
    add_kept(c, "x", "x_scales", a.x, a.x_scales, a.m, a.k, a.x_stride, a.x_scales_stride, a.dtype, a.dgate_weight && a.n > 0, false);
    c.add("gate_weight", a.gate_weight, a.n, a.k, a.gate_weight_stride, a.dtype, a.dx && a.m > 0);
    c.add("up_weight", a.up_weight, a.n, a.k, a.up_weight_stride, a.dtype, a.dx && a.m > 0);
    add_kept(c, "gate", "gate_scales", a.gate, a.gate_scales, a.m, a.n, a.gate_stride, a.gate_scales_stride, a.dtype, any, false);
    add_kept(c, "up", "up_scales", a.up, a.up_scales, a.m, a.n, a.up_stride, a.up_scales_stride, a.dtype, any, false);
    c.add("out", a.out, a.m, a.n, a.out_stride, a.dtype, false, true, a.dout);
    c.add("dx", a.dx, a.m, a.k, a.dx_stride, a.dtype, false, true);
    c.add("dgate_weight", a.dgate_weight, a.n, a.k, a.dgate_weight_stride, a.dtype, false, true);
    c.add("dup_weight", a.dup_weight, a.n, a.k, a.dup_weight_stride, a.dtype, false, true);
    return c.done();
}

fsdp_status ready_gated(const fsdp_step_gated_grad_args& a, Grad& g) {
    fsdp_status st = check_gated_grad(a);
    if (st != FSDP_OK) return st;
    g.m = a.m;
    g.n = a.n;
    g.k = a.k;
    g.dtype = a.dtype;
    g.two = true;
    g.dx = a.dx;
    g.dweight = a.dgate_weight;
    g.saved_x = a.x_scales;
    g.weight[0] = {a.gate_weight, a.n, a.k, row_stride(a.n, a.k, a.gate_weight_stride), false};
    g.weight[1] = {a.up_weight, a.n, a.k, row_stride(a.n, a.k, a.up_weight_stride), false};
    g.x = {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false};
    shape_grad(g);
    if ((st = check_reach(g)) != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    plan_grad(g, cus, a.dx || a.dgate_weight, false);
    return FSDP_OK;
}

fsdp_status check_linear_grad(const fsdp_step_linear_grad_args& a) {
    const fsdp_status st = check_sizes(a.m, a.n, 1, a.k, a.dtype, a.activation);
    if (st != FSDP_OK) return st;
    const bool any = a.dx || a.dweight || a.dbias || a.dtimes;
    const bool slopes = a.dx || a.dweight || a.dbias;
    if (a.dtimes && !a.times && a.m > 0) return fail(FSDP_ERR_INVALID, "dtimes needs times");
    Checked c;
    c.add_in_place("dout", a.dout, a.m, a.n, a.dout_stride, a.dtype, any);
    add_kept(c, "x", "x_scales", a.x, a.x_scales, a.m, a.k, a.x_stride, a.x_scales_stride, a.dtype, a.dweight && a.n > 0, false);
    c.add("weight", a.weight, a.n, a.k, a.weight_stride, a.dtype, a.dx && a.m > 0);
    add_kept(c, "pre", "pre_scales", a.pre, a.pre_scales, a.m, a.n, a.pre_stride, a.pre_scales_stride, a.dtype,
             a.dtimes || (slopes && a.activation != FSDP_ACT_NONE), false);
    c.add_in_place("times", a.times, a.m, a.n, a.times_stride, a.dtype, false);
    c.add("dx", a.dx, a.m, a.k, a.dx_stride, a.dtype, false, true);
    c.add("dweight", a.dweight, a.n, a.k, a.dweight_stride, a.dtype, false, true);
    c.add_vector("dbias", a.dbias, a.n, a.dtype, false, true);
    c.add("dtimes", a.dtimes, a.m, a.n, a.dtimes_stride, a.dtype, false, true, a.times);
    return c.done();
}

fsdp_status ready_linear(const fsdp_step_linear_grad_args& a, Grad& g) {
    fsdp_status st = check_linear_grad(a);
    if (st != FSDP_OK) return st;
    g.m = a.m;
    g.n = a.n;
    g.k = a.k;
    g.dtype = a.dtype;
    g.dx = a.dx;
    g.dweight = a.dweight;
    g.saved_x = a.x_scales;
    g.weight[0] = {a.weight, a.n, a.k, row_stride(a.n, a.k, a.weight_stride), false};
    g.as_is = !a.times && a.activation == FSDP_ACT_NONE;
    g.dout = {a.dout, a.m, a.n, row_stride(a.m, a.n, a.dout_stride), false};
    g.x = {a.x, a.m, a.k, row_stride(a.m, a.k, a.x_stride), false};
    shape_grad(g);
    if ((st = check_reach(g)) != FSDP_OK) return st;
    const int cus = cu_count(&st);
    if (cus == 0) return st;
    plan_grad(g, cus, a.dx || a.dweight, a.dbias);
    return FSDP_OK;
}

}  // namespace
}  // namespace fsdp_block

using namespace fsdp_block;

extern "C" fsdp_status fsdp_step_gated_workspace(const fsdp_step_gated_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    Forward f;
    const fsdp_status st = ready_forward(*args, f);
    if (st == FSDP_OK) *bytes = f.bytes;
    return st;
}

extern "C" fsdp_status fsdp_step_gated(const fsdp_step_gated_args* args, void* workspace, int64_t workspace_bytes,
                                       hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_step_gated_args& a = *args;
    Forward f;
    fsdp_status st = ready_forward(a, f);
    if (st != FSDP_OK) return st;
    if ((st = check_workspace(workspace, workspace_bytes, f.bytes)) != FSDP_OK) return st;
    if (a.m == 0 || a.n == 0) return FSDP_OK;
    char* const ws = static_cast<char*>(workspace);
    PairProduct p{};
    p.a = a.x;
    p.a_stride = f.x.stride;
    p.b = a.gate_weight;
    p.b_stride = f.gate.stride;
    p.b2 = a.up_weight;
    p.b2_stride = f.up.stride;
    p.m = a.m;
    p.n = 2 * a.n;
    p.k = a.k;
    p.inner = a.n;
    p.e.act = a.activation;
    p.e.out = a.out;
    p.e.out_stride = a.out_stride;
    p.gate = a.gate;
    p.gate_scales = static_cast<uint8_t*>(a.gate_scales);
    p.gate_stride = a.gate_stride;
    p.gate_scales_stride = a.gate_scales_stride;
    p.up = a.up;
    p.up_scales = static_cast<uint8_t*>(a.up_scales);
    p.up_stride = a.up_stride;
    p.up_scales_stride = a.up_scales_stride;
    if (by_rows(a, f.shape))
        return with_type(a.dtype, [&](auto type) {
            using T = decltype(type);
            const auto rows = [&](auto count) {
                constexpr int kRows = decltype(count)::value;
                // One wave to a SIMD and less, and a row of several steps for each of four.
                const int64_t waves = ceil_div(a.n, kGatedOut<kRows>);
                if (waves <= 4 * int64_t(f.cus) && a.k >= 4096) return launch(gated_row_kernel<T, kRows, true>, p, dim3(unsigned(waves)), 256, stream);
                return launch(gated_row_kernel<T, kRows, false>, p, dim3(unsigned(ceil_div(waves, 4))), 256, stream);
            };
            return a.m == 1   ? rows(std::integral_constant<int, 1>())
                   : a.m == 2 ? rows(std::integral_constant<int, 2>())
                              : rows(std::integral_constant<int, 4>());
        });
    Pads<3> pads;
    const auto lay = [&](const Source& o, int64_t at, const void** to, int64_t* stride) {
        if (at < 0) return;
        pads.add(o, a.dtype, ws + at);
        *to = ws + at;
        *stride = lined(o.cols, a.dtype);
    };
    lay(f.x, f.pad[0], &p.a, &p.a_stride);
    lay(f.gate, f.pad[1], &p.b, &p.b_stride);
    lay(f.up, f.pad[2], &p.b2, &p.b2_stride);
    if ((st = pads.run(stream)) != FSDP_OK) return st;
    return run_pair<GatedForward>(p, f.cut, a.dtype, ws, stream);
}

extern "C" fsdp_status fsdp_step_gated_grad_workspace(const fsdp_step_gated_grad_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    Grad g;
    const fsdp_status st = ready_gated(*args, g);
    if (st == FSDP_OK) *bytes = g.bytes;
    return st;
}

extern "C" fsdp_status fsdp_step_gated_grad(const fsdp_step_gated_grad_args* args, void* workspace, int64_t workspace_bytes,
                                            hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_step_gated_grad_args& a = *args;
    Grad g;
    fsdp_status st = ready_gated(a, g);
    if (st != FSDP_OK) return st;
    if ((st = check_workspace(workspace, workspace_bytes, g.bytes)) != FSDP_OK) return st;
    char* const ws = static_cast<char*>(workspace);
    if (a.m > 0 && a.n > 0 && (g.dz >= 0 || a.out)) {
        const GatedSlopeArgs s{a.dout, a.gate, a.up, static_cast<const uint8_t*>(a.gate_scales), static_cast<const uint8_t*>(a.up_scales),
                               g.dz >= 0 ? ws + g.dz : nullptr, a.out, a.dout_stride, a.gate_stride, a.up_stride, a.gate_scales_stride,
                               a.up_scales_stride, g.wide, a.out_stride, a.m, a.n, g.split, g.part_rows, a.activation};
        const dim3 grid(unsigned(ceil_div(g.split, 512)), unsigned(g.row_parts));
        st = with_type(a.dtype, [&](auto type) {
            using T = decltype(type);
            return a.gate_scales ? launch(gated_slope_kernel<T, true>, s, grid, 256, stream)
                                 : launch(gated_slope_kernel<T, false>, s, grid, 256, stream);
        });
        if (st != FSDP_OK) return st;
    }
    return run_products(g, a.x, a.x_scales, a.x_scales_stride, a.dx, a.dx_stride, a.dgate_weight, a.dgate_weight_stride, a.dup_weight,
                        a.dup_weight_stride, ws, stream);
}

extern "C" fsdp_status fsdp_step_linear_grad_workspace(const fsdp_step_linear_grad_args* args, int64_t* bytes) {
    clear_error();
    if (!args || !bytes) return fail(FSDP_ERR_INVALID, "args or bytes is NULL");
    Grad g;
    const fsdp_status st = ready_linear(*args, g);
    if (st == FSDP_OK) *bytes = g.bytes;
    return st;
}

extern "C" fsdp_status fsdp_step_linear_grad(const fsdp_step_linear_grad_args* args, void* workspace, int64_t workspace_bytes,
                                             hipStream_t stream) {
    clear_error();
    if (!args) return fail(FSDP_ERR_INVALID, "args is NULL");
    const fsdp_step_linear_grad_args& a = *args;
    Grad g;
    fsdp_status st = ready_linear(a, g);
    if (st != FSDP_OK) return st;
    if ((st = check_workspace(workspace, workspace_bytes, g.bytes)) != FSDP_OK) return st;
    char* const ws = static_cast<char*>(workspace);
    float* const sums = g.sums < 0 ? nullptr : reinterpret_cast<float*>(ws + g.sums);
    char* const dz = g.dz >= 0 && !g.as_is ? ws + g.dz : nullptr;
    if (a.m > 0 && a.n > 0 && (dz || sums || a.dtimes)) {
        const SavedSlopeArgs s{a.dout, a.pre, a.times, static_cast<const uint8_t*>(a.pre_scales), dz, a.dtimes, sums, a.dout_stride,
                               a.pre_stride, a.pre_scales_stride, a.times_stride, g.wide, a.dtimes_stride, a.m, a.n, g.split, g.part_rows,
                               a.activation};
        const dim3 grid(unsigned(ceil_div(g.split, 512)), unsigned(g.row_parts));
        st = with_type(a.dtype, [&](auto type) {
            using T = decltype(type);
            return a.pre_scales ? launch(saved_slope_kernel<T, true>, s, grid, 256, stream)
                                : launch(saved_slope_kernel<T, false>, s, grid, 256, stream);
        });
        if (st != FSDP_OK) return st;
    }
    Join j(int(a.n));
    j.add(a.dbias, sums, g.row_parts, a.dbias ? 1 : 0, a.dtype);
    if ((st = j.run(a.dtype, stream)) != FSDP_OK) return st;
    return run_products(g, a.x, a.x_scales, a.x_scales_stride, a.dx, a.dx_stride, a.dweight, a.dweight_stride, nullptr, 0, ws, stream);
}
