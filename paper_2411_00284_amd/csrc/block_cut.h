// How a matrix product is run (host code): in which tiles, in how many parts of
// k, in one launch or two, and which operands are laid on the grid first.
#pragma once

#include "block_device.h"
#include "block_host.h"

#include <algorithm>

namespace fsdp_block {
namespace {

template <typename F>
fsdp_status with_type(fsdp_dtype dtype, F f) {
    return dtype == FSDP_DTYPE_BF16 ? f(bf16(0.f)) : dtype == FSDP_DTYPE_F16 ? f(f16(0.f)) : f(0.f);
}

// The forms of a product in tiles.  Times in us of a step (64 k, fp32: 32) on one
// MI355X: `alone` with one workgroup on a CU, `full` with `held` of them on every
// CU, and `fixed` for the start and the end of a tile, as measured over products from
// 16 x 14336 x 4096 to 8192 x 28672 x 8192.  A guide, not a prediction: 64 x 64 tiles
// of 771 x 1153 x 2501 take 0.4 us a step.  Those of fp32 are from 2048 x 1024 x 688 and
// 4096^3 only: dx of the former is expected at 24 us and takes 33.
struct Form {
    int tile_m, tile_n, steps, held;
    double alone, full, fixed;
};
constexpr Form kForms16[] = {
    {256, 256, 2, 1, 1.15, 1.60, 6.0},
    {128, 128, 2, 2, 0.60, 0.97, 4.0},
    {128, 128, 4, 1, 0.36, 0.52, 3.5},
    {64, 128, 4, 1, 0.25, 0.32, 3.5},
    {64, 64, 8, 1, 0.14, 0.20, 3.5},
};
constexpr Form kForms32[] = {
    {128, 128, 2, 2, 1.80, 3.60, 4.0},
    {64, 128, 4, 1, 0.95, 0.95, 3.5},
};

// The forms that a library has, the smallest last, and those that the rest of a last round
// may go in.
struct Forms {
    const Form* all;
    int count;
    const Form* rest;
    int rests;
};
constexpr Forms kLinear16{kForms16, 5, kForms16 + 1, 1}, kLinear32{kForms32, 2, nullptr, 0};
inline const Forms& linear_forms(fsdp_dtype dtype) { return dtype == FSDP_DTYPE_F32 ? kLinear32 : kLinear16; }

// How one product is run.
struct Cut {
    const Form* form = nullptr;      // NULL: row_kernel
    int count = 1;                   // parts of k
    int64_t part_k = 0;
    // Not NULL: the rows (columns) of out from rest_at on are a launch of their own.
    const Form* rest = nullptr;
    bool rest_rows = false;
    int64_t rest_at = 0;
    // Byte offsets in the workspace and its size: the operands laid on the grid, the parts.
    int64_t pad_a = -1, pad_b = -1, parts = -1, bytes = 0;
};

struct Shape {
    int64_t m, n, k;
    fsdp_dtype dtype;
    bool columns_a, columns_b;
    int64_t stride_a, stride_b;      // of the operands as they are laid on the grid
};

// The most bytes that a load may lie from its tile's first (Operand::load), and
// whether a form's loads stay within: an operand by rows has the tile's rows in a
// step, one by columns the step's rows of k.
constexpr int64_t kReach = 0x7ffffff0;
bool reaches(const Form& f, const Shape& s) {
    const int64_t size = elem_bytes(s.dtype), deep = 128 / size;
    const auto end = [&](bool columns, int64_t rows, int64_t tile, int64_t stride) {
        return columns ? ((std::min(deep, s.k) - 1) * stride + tile) * size : (std::min(tile, rows) - 1) * stride * size + 128;
    };
    return end(s.columns_a, s.m, f.tile_m, s.stride_a) <= kReach && end(s.columns_b, s.n, f.tile_n, s.stride_b) <= kReach;
}

constexpr int64_t kMostRows = 4;     // of row_kernel
// Below 2^27 columns: eight or sixteen of them to a workgroup must make fewer than 2^32 threads.
bool row_form(const Shape& s) { return s.m <= kMostRows && s.n < (int64_t(1) << 27) && !s.columns_a && !s.columns_b; }

// Bytes per us in which the operands come out of memory, in all and to one
// workgroup, and what the caches keep of them: with the second bound, which wants
// 220 workgroups, 64 x 14336 -> 4096 takes 29.5 us instead of 45, 64 x 28672 -> 8192
// 104 instead of 140; under 16 MB it would cut products for nothing (64 x 1024 -> 1024
// 9.1 us instead of 7.2).
constexpr double kMostRead = 5.5e6, kGroupRead = 0.025e6, kCached = 16e6;

// Of whole rounds of workgroups and the last one.
double rounds_time(const Form& form, int64_t groups, int64_t steps, int cus) {
    const int64_t slots = int64_t(cus) * form.held, whole = groups / slots, rest = groups - whole * slots;
    const double time = double(whole) * (double(steps) * form.full + form.fixed);
    return rest ? time + double(steps) * (rest > cus ? form.full : form.alone) + form.fixed : time;
}

// The form and the cut with the least expected time: whole rounds of workgroups
// over the CUs, the fullest CU of the last round, reading the operands if that takes
// longer, and the join of the parts (3 us, and 8 bytes moved per value and part).
// Up to four rows of x, row_kernel reads the weight at HBM's rate in one launch.
// Tiles of 256 x 256 that leave a last round of few are cut where the whole rounds
// end, and the rest of out takes tiles of 128 x 128 in a second launch (3 us): bf16
// 6144 x 6144 x 4096 takes 281 us instead of 301, 14336 x 4096 with k = 8192 746
// instead of 791.  (Smaller tiles for the rest: 334 instead of 300 us at 5000^3.)
// `rows_too`: up to four rows go without tiles.
Cut choose(const Shape& s, int cus, const Forms& set, bool rows_too = true) {
    Cut best;
    if (rows_too && row_form(s)) return best;
    const bool wide = s.dtype == FSDP_DTYPE_F32;
    const int step_k = wide ? 32 : 64;
    const int64_t steps = std::max<int64_t>(1, ceil_div(s.k, step_k));
    const double read = double(elem_bytes(s.dtype)) * (double(s.m) * double(s.k) + double(s.n) * double(s.k));
    const double joining = double(s.m) * double(s.n) * 8 / 5e6;
    double least = 0;
    for (int f = 0; f < set.count; ++f) {
        const Form& form = set.all[f];
        if (!reaches(form, s)) continue;
        const int64_t tiles = ceil_div(s.m, form.tile_m) * ceil_div(s.n, form.tile_n);
        for (int parts = 1; parts <= 16; ++parts) {
            // Parts of at least four steps, and no more of them than some rounds.
            if (parts > 1 && (steps < 4 * parts || tiles * (parts - 1) > 3 * int64_t(cus))) break;
            const int64_t each = (steps + parts - 1) / parts, count = (steps + each - 1) / each;
            if (count != parts) continue;
            const int64_t groups = tiles * parts;
            double time = rounds_time(form, groups, each, cus);
            const double rate = read > kCached ? std::min(kMostRead, kGroupRead * double(groups)) : kMostRead;
            time = std::max(time, read / rate + form.fixed);
            if (parts > 1) time += 3.0 + double(parts) * joining;
            if (!best.form || time < least) {
                least = time;
                best.form = &form;
                best.part_k = each * step_k;
                best.count = parts;
            }
        }
    }
    if (set.rests == 0 || s.m == 0 || s.n == 0) return best;
    const Form& big = set.all[0];
    if (!reaches(big, s)) return best;
    const int64_t down = ceil_div(s.m, big.tile_m), across = ceil_div(s.n, big.tile_n);
    for (const bool rows : {true, false}) {
        // Rows (columns) of tiles in whole rounds, and what is left of out.
        const int64_t other = rows ? across : down, taken = down * across / cus * cus / other;
        const int64_t at = taken * (rows ? big.tile_m : big.tile_n), m = rows ? s.m - at : s.m, n = rows ? s.n : s.n - at;
        if (taken == 0 || m <= 0 || n <= 0) continue;
        for (int f = 0; f < set.rests; ++f) {
            const Form& small = set.rest[f];
            const double time = rounds_time(big, taken * other, steps, cus) + 3.0 +
                                rounds_time(small, ceil_div(m, small.tile_m) * ceil_div(n, small.tile_n), steps, cus);
            if (time >= least) continue;
            least = time;
            best = Cut{};
            best.form = &big;
            best.part_k = steps * step_k;
            best.rest = &small;
            best.rest_rows = rows;
            best.rest_at = at;
        }
    }
    return best;
}

struct Source {
    const void* p;
    int64_t rows, cols, stride;      // as it lies in memory
    bool zeros;                      // zeros follow a row, up to a whole 16-byte unit
};

// Elements of a row laid out in whole lines.
int64_t lined(int64_t cols, fsdp_dtype dtype) { return round_up(cols, 128 / elem_bytes(dtype)); }

// Whether an operand lies on the 16-byte grid in whole units, as product_kernel
// reads it, with the offsets of a step in 31 bits.
bool on_grid(const Source& o, fsdp_dtype dtype) {
    const int unit = 16 / elem_bytes(dtype);
    return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && o.stride % unit == 0 && o.stride < (1 << 21) && (o.zeros || o.cols % unit == 0);
}

// A row's stride where product_kernel reads it.
int64_t laid_stride(const Source& o, fsdp_dtype dtype) { return on_grid(o, dtype) ? o.stride : lined(o.cols, dtype); }

// Whether any form reaches the operands (row_kernel reaches all of its).
fsdp_status check_reach(const Shape& s, const Forms& set, bool rows_too = true) {
    if (s.m == 0 || s.n == 0 || (rows_too && row_form(s))) return FSDP_OK;
    if (reaches(set.all[set.count - 1], s)) return FSDP_OK;
    return fail(FSDP_ERR_OVERFLOW, "a tile's rows of an operand of %lld x %lld, %lld x %lld do not lie within 2^31 bytes",
                (long long)s.m, (long long)s.k, (long long)s.n, (long long)s.k);
}

}  // namespace
}  // namespace fsdp_block
