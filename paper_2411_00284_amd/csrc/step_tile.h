// Matrix products of 16-bit operands in tiles of 256 x 256 and 128 x 128
// (block_product.h has the others): out[i][j] = sum_k A[i][k] B[j][k], an operand by
// rows or by columns as there.
//
// A tile belongs to four waves, each a quarter of it, in 16 x 16 x 32 matrix
// instructions, which run at 1960 TFLOP/s alone where those of 32 x 32 x 16 run at 1710
// (one MI355X, normal values: at the clock that its power leaves).
//
// k goes by in steps of 64, a line of 128 bytes a row. Both operands of a step lie in a
// ring of kRing places in LDS: A and B of a step, those of the next, and what is on its
// way. A step is worked on in two halves of 32 k, whose operands lie in registers: while the
// matrix cores take one half, the registers of the next are read, and of one operand the
// loads from memory to LDS are issued. Once the second half is in registers (a
// barrier) the step's places are free. So each half issues one operand's loads, four
// matrix instructions apart: a wave is alone on its SIMD, and while it waits to issue a load it
// issues no matrix instruction (all loads of a step in one half: 1360 instead of 1420
// TFLOP/s at 8192 x 8192 x 4096, 1400 instead of 1500 at 8192 x 4096 x 14336; 32 x 32
// instructions in the schedule of block_product.h: 1090 and 1290). With zeros for
// values, which take little power, the loop runs at 1740 to 1830: what bounds it is power.
//
// The accumulators fill all 256 accumulation registers. The compiler gives a matrix
// instruction another destination than its addend if it may, and then has none left: so
// the instruction is written out with one register for both, and the loop ends in a wait for
// what the compiler cannot know of (the results' latency). tests/test_step_isa.py looks
// that no instruction of the loop itself comes too near to one of these.
#pragma once

#include "block_product.h"

namespace fsdp_block {
namespace {

typedef float Acc4 __attribute__((ext_vector_type(4)));

// c += a b: lane l has row l % 16 of both and the (l / 16)-th 16 bytes of a 64-byte run
// of k; element r of c is at A row 4 (l / 16) + r, B row l % 16.
__device__ __forceinline__ void mma16(Eight<bf16> a, Eight<bf16> b, Acc4& c) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mma16(Eight<f16> a, Eight<f16> b, Acc4& c) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// Nothing that follows reads the sums before the matrix cores have written them.
template <int kN>
__device__ __forceinline__ void settle(Acc4 (&c)[kN][kN]) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
    for (int x = 0; x < kN; ++x)
#pragma unroll
        for (int y = 0; y < kN; y += 4) asm volatile("" : "+a"(c[x][y]), "+a"(c[x][y + 1]), "+a"(c[x][y + 2]), "+a"(c[x][y + 3]));
    __builtin_amdgcn_sched_barrier(0);
}

// An operand's loads. LDS holds "rows" as 128 bytes per row with the 16-byte units of row
// r exchanged by r / 2, "columns" as a run of columns per k with its units exchanged by
// exchange(k); both are read without conflicts.
template <typename T, int kRows, bool kColumns>
struct Stream {
    static constexpr int kBytes = kRows * 128, kLoads = kRows / 32, kUnits = kRows / 8;
    static constexpr int64_t kNowhere = 0xfffffff0u;   // out of any range
    static constexpr uint32_t kMost = 0x7ffffff0u;
    __device__ static __forceinline__ int exchange(int k) { return (k & 3) * 4 + (k >> 3 & 1) * 2; }

    const char* at;            // the next step's first byte
    int64_t step, left;        // bytes to the step after it, and to the operand's end, in whole units
    int rest;                  // k not yet asked for
    uint32_t offset[kLoads];
    int k;                     // this lane's first k of a step ("rows")
    __amdgpu_buffer_rsrc_t from;

    __device__ __forceinline__ void begin_at(const void* p, int64_t stride, int64_t first, int64_t rows, int64_t k0, int64_t k1) {
        if constexpr (kColumns) {
            at = static_cast<const char*>(p) + (k0 * stride + first) * 2;
            step = 128 * stride;
            left = (k1 - 1 - k0) * stride * 2 + (rows - first + 7) / 8 * 16;
        } else {
            at = static_cast<const char*>(p) + (first * stride + k0) * 2;
            step = 128;
            left = (rows - 1 - first) * stride * 2 + (k1 - k0 + 7) / 8 * 16;
        }
    }
    __device__ __forceinline__ Stream(const void* p, int64_t stride, int64_t first, int64_t rows, int64_t k0, int64_t k1) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        begin_at(p, stride, first, rows, k0, k1);
        rest = int(k1 - k0);
        k = (lane % 8 ^ (wave % 2 * 4 + lane / 16)) * 8;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            if constexpr (kColumns) {
                const int unit = (j * 4 + wave) * 64 + lane, kk = unit / kUnits, u = unit % kUnits;
                offset[j] = uint32_t(min(kk * stride * 2 + (u ^ exchange(kk)) * 16, kNowhere));
            } else {
                offset[j] = uint32_t(min(((j * 4 + wave) * 8 + lane / 8) * stride * 2 + k * 2, kNowhere));
            }
        }
    }
    // (`bytes` is not negative while there is something to ask for; what passes 31 bits is out of any tile's reach.)
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t range(const char* p, int64_t bytes) const {
        const uint32_t n = uint64_t(bytes) >> 31 ? kMost : uint32_t(bytes);
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, int(rest <= 0 ? 0u : n), 0x00020000);
    }
    // Units of the last step that lie past k are asked for out of range, and so are zeros.
    __device__ __forceinline__ void cut() {
        if (!kColumns && rest < 64)
#pragma unroll
            for (int j = 0; j < kLoads; ++j) offset[j] = k < rest ? offset[j] : uint32_t(kNowhere);
    }
    // The loads that follow are the next step's.
    __device__ __forceinline__ void next() {
        cut();
        from = range(at, left);
        at += step;
        left -= step;
        rest -= 64;
    }
    // `own`: 1024 times the wave.
    __device__ __forceinline__ void load(char* lds, int j, int own) const {
        typedef __attribute__((address_space(3))) void lds_void;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)(lds + j * 4096 + own), 16, int(offset[j]), 0, 0, 0);
    }
};

// A wave's registers of half a step: kTiles times 16 rows of an operand. kApart: how many
// rows lie between the first half of the tiles and the second, over what they cover.
// kWoven ("rows"): tiles 2 y and 2 y + 1 have 32 rows in turns of four, tile 2 y the first four of
// each eight; LDS then exchanges the units of row r by (r / 8 % 4) * 2 + r / 2 % 2.
template <typename T, int kRows, bool kColumns, int kTiles, int kApart, bool kWoven = false>
struct Half {
    static constexpr int kPlaces = kColumns ? kTiles : 2;
    Eight<T> v[kTiles];
    __device__ static __forceinline__ void lane_places(int first, int (&place)[kPlaces]) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int x = 0; x < kPlaces; ++x) {
            if constexpr (kWoven) {
                place[x] = (first + lane % 16 / 4 * 8 + lane % 4) * 128 + ((4 * x + lane / 16) ^ (lane % 16 / 4 * 2 + lane % 4 / 2)) * 16;
            } else if constexpr (!kColumns) {
                place[x] = (first + lane % 16) * 128 + ((4 * x + lane / 16) ^ lane / 2 % 8) * 16;
            } else {
                // The 4 x 16 block of k and columns that 16 lanes point to; k + 4 and k + 32 are exchanged alike.
                const int k = lane / 16 * 8 + lane % 16 / 4, byte = (first + 16 * x + lane % 4 * 4) * 2;
                place[x] = k * kRows * 2 + (byte ^ Stream<T, kRows, true>::exchange(k) * 16);
            }
        }
    }
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    static constexpr int kReads = kColumns ? 2 * kTiles : kTiles;      // LDS instructions
    s16x4 low;                       // the first of two
    // Read `i` of kReads, in order.
    __device__ __forceinline__ void read(const char* lds, const int (&place)[kPlaces], int half, int i) {
        if constexpr (!kColumns) {
            const int row = (kWoven ? i / 2 * 32 + i % 2 * 4 : i * 16) + (i >= kTiles / 2 ? kApart : 0);
            v[i] = *reinterpret_cast<const Eight<T>*>(lds + place[half] + row * 128);
        } else {
            // The transposing load gives lane i of 16 the i-th column of their block.
            const int x = i / 2;
            const s16x4 got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + place[x] + half * 32 * kRows * 2 + i % 2 * 4 * kRows * 2));
            if (i % 2 == 0) low = got;
            else v[x] = __builtin_bit_cast(Eight<T>, __builtin_shufflevector(low, got, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

template <typename T, bool kColumnsA, bool kColumnsB, int kTile, int kRing, typename Kind, typename Args>
__device__ __forceinline__ void ring_tile(const Args& p) {
    using A = Stream<T, kTile, kColumnsA>;
    using B = typename Kind::template Ring<T, kTile, kColumnsB>;
    constexpr int kN = kTile / 32, kLoads = A::kLoads, kBytes = A::kBytes, kPeriod = 5;
    static_assert(kRing == 5 || kRing == 10, "places that come round in kPeriod steps");
    constexpr int kMore = kRing > 5 ? kBytes : 16;
    // One array per place: their reads and loads are known not to touch each other.
    __shared__ __attribute__((aligned(1024))) char r0[kBytes], r1[kBytes], r2[kBytes], r3[kBytes], r4[kBytes], r5[kMore], r6[kMore],
        r7[kMore], r8[kMore], r9[kMore];
    char* const ring[10] = {r0, r1, r2, r3, r4, r5, r6, r7, r8, r9};
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave / 2 * (kTile / 2), wj = wave % 2 * (kTile / 2);
    const TilePlace t = tile_place(blockIdx.x, unsigned((p.m - p.first_i + kTile - 1) / kTile), unsigned((p.n - p.first_j + kTile - 1) / kTile),
                                   unsigned(p.count));
    const int64_t i0 = p.first_i + int64_t(t.row) * kTile, j0 = p.first_j + int64_t(t.column) * kTile;
    const int64_t k0 = t.part * p.part_k, k1 = min(k0 + p.part_k, p.k);
    A a(p.a, p.a_stride, i0, p.m, k0, k1);
    B b = Kind::template ring_operand<T, kTile, kColumnsB>(p, j0, k0, k1);
    using FA = Half<T, kTile, kColumnsA, kN, 0>;
    using FB = Half<T, kTile, kColumnsB, kN, Kind::kPair ? kTile / 4 : 0, Kind::kPair>;
    FA fa[2];
    FB fb[2];
    int pa[FA::kPlaces], pb[FB::kPlaces];
    FA::lane_places(wi, pa);
    FB::lane_places(Kind::kPair ? wj / 2 : wj, pb);
    Acc4 acc[kN][kN];
#pragma unroll
    for (int x = 0; x < kN; ++x)
#pragma unroll
        for (int y = 0; y < kN; ++y) acc[x][y] = Acc4{0.f, 0.f, 0.f, 0.f};

    // Waits for this wave's loads, but for those of the last kLater operands, and its LDS
    // reads; then for the other waves.
    const auto sync = [](auto later) {
        constexpr int n = decltype(later)::value * kLoads;
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 7 << 4);        // vmcnt(n) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // The q-th operand of all (A of step q / 2 for even q, else B) to its place.
    const auto ask = [&](auto q, int j, int own) {
        constexpr int kQ = decltype(q)::value;
        if constexpr (kQ % 2 == 0) a.load(ring[kQ % kRing], j, own);
        else b.load(ring[kQ % kRing], j, own);
    };
    const auto next = [&](auto q) {
        if constexpr (decltype(q)::value % 2 == 0) a.next();
        else b.next();
    };
    // The matrix instructions of the half in registers `kS`, the reads of the other half (half
    // kS ^ 1 of the step whose A is the kQ-th operand), the loads of operand kAsk; in this order.
    const auto half = [&](auto s, auto q, auto asked) {
        constexpr int kS = decltype(s)::value, kQ = decltype(q)::value, kAll = kN * kN;
        // Both operands' reads, one after each of the first half of the matrix instructions (or each
        // second one of them, if there are as few); the loads between them, or after them.
        constexpr int kReads = FA::kReads + FB::kReads, kGap = kReads * 4 <= kAll ? 2 : 1;
        constexpr bool kBetween = kGap == 2;
        constexpr int kFirst = kBetween ? 1 : kAll / 2, kEvery = kAll / 2 / kLoads;
        int own = wave * 1024;
        asm volatile("" : "+s"(own));            // an addition a load, instead of a register for each place and load
#pragma unroll
        for (int i = 0; i < kAll; ++i) {
            if (i % kGap == 0 && i / kGap < kReads) {
                constexpr int kFew = FA::kReads < FB::kReads ? FA::kReads : FB::kReads;
                // In turn, as long as there are two.
                const int r = i / kGap, a_reads = r < 2 * kFew ? (r + 1) / 2 : FA::kReads > kFew ? r - kFew : kFew;
                const bool from_a = r < 2 * kFew ? r % 2 == 0 : FA::kReads > kFew;
                __builtin_amdgcn_sched_barrier(0);
                if (from_a) fa[kS ^ 1].read(ring[kQ % kRing], pa, kS ^ 1, a_reads);
                else fb[kS ^ 1].read(ring[(kQ + 1) % kRing], pb, kS ^ 1, r - a_reads);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (i >= kFirst && (i - kFirst) % kEvery == 0 && (i - kFirst) / kEvery < kLoads) {
                __builtin_amdgcn_sched_barrier(0);
                ask(asked, (i - kFirst) / kEvery, own);
                __builtin_amdgcn_sched_barrier(0);
            }
            // A pair's sums lie the other way round: a lane has a row of A and, of two woven tiles of B, eight
            // neighbouring columns.
            if constexpr (Kind::kPair) mma16(fb[kS].v[i % kN], fa[kS].v[i / kN], acc[i / kN][i % kN]);
            else mma16(fa[kS].v[i / kN], fb[kS].v[i % kN], acc[i / kN][i % kN]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Step s of a period: operands 2 s and 2 s + 1; kRing operands are in LDS or on their way.
    const auto step = [&](auto s) {
        constexpr int kQ = 2 * decltype(s)::value;
        using First = std::integral_constant<int, kQ + kRing - 1>;
        using Second = std::integral_constant<int, kQ + kRing>;
        next(First());
        half(std::integral_constant<int, 0>(), std::integral_constant<int, kQ>(), First());
        next(Second());
        sync(std::integral_constant<int, kRing - 4>());
        half(std::integral_constant<int, 1>(), std::integral_constant<int, kQ + 2>(), Second());
    };
    const auto start = [&](auto q) {
        next(q);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) ask(q, j, wave * 1024);
    };
    start(std::integral_constant<int, 0>());
    start(std::integral_constant<int, 1>());
    start(std::integral_constant<int, 2>());
    start(std::integral_constant<int, 3>());
    if constexpr (kRing > 5) {
        start(std::integral_constant<int, 4>());
        start(std::integral_constant<int, 5>());
        start(std::integral_constant<int, 6>());
        start(std::integral_constant<int, 7>());
        start(std::integral_constant<int, 8>());
    }
    sync(std::integral_constant<int, kRing - 3>());
#pragma unroll
    for (int r = 0; r < FA::kReads; ++r) fa[0].read(r0, pa, 0, r);
#pragma unroll
    for (int r = 0; r < FB::kReads; ++r) fb[0].read(r1, pb, 0, r);
    // Steps past the end add zeros: the loop takes a period at a time.
    for (int left = int(k1 - k0); left > 0; left -= 64 * kPeriod) {
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
        step(std::integral_constant<int, 4>());
        settle(acc);
    }
    settle(acc);
    sync(std::integral_constant<int, 0>());                       // nothing more is written to LDS

    if constexpr (Kind::kPair) {
        // A lane finishes what it holds, a row's 64 bytes of four lanes at a time. It passes the sums through
        // LDS all the same, its own only: so that the code of the columns is there once. A tile that lies in
        // out whole takes two rows (and two groups of a row) together: with one wave on a SIMD the chains of
        // one alone leave it waiting (4096 x 14336 x 1024 kept in 8 bits: 364 us instead of 417; with k = 4096
        // and 2048 rows, and two restores of 22 us after it, 433 instead of 450).
        typedef Acc4 Acc4x64[64];
        static_assert(4 * kN * sizeof(Acc4x64) <= kBytes);
        Acc4x64* const mine = reinterpret_cast<Acc4x64*>(wave == 0 ? r0 : wave == 1 ? r1 : wave == 2 ? r2 : r3);
        const int64_t i = i0 + wi + lane % 16, j = (j0 + wj) / 2 + lane / 16 * 8;
        const bool whole = Kind::whole(p, i0, j0 / 2, kTile);
        const auto fetch = [&](int x, int y, float (&g)[8], float (&u)[8]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Acc4 gh = mine[x * kN + y + h][lane], uh = mine[x * kN + kN / 2 + y + h][lane];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    g[4 * h + c] = gh[c];
                    u[4 * h + c] = uh[c];
                }
            }
        };
#pragma unroll
        for (int x0 = 0; x0 < kN; x0 += 4) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < kN; ++y) mine[x * kN + y][lane] = acc[x0 + x][y];
            if (whole) {
                constexpr int kDown = 2, kAcross = kN / 4;
#pragma unroll 1
                for (int x = 0; x < 4; x += kDown) {
                    float g[kDown][kAcross][8], u[kDown][kAcross][8];
#pragma unroll
                    for (int d = 0; d < kDown; ++d)
#pragma unroll
                        for (int a = 0; a < kAcross; ++a) fetch(x + d, 2 * a, g[d][a], u[d][a]);
                    Kind::template put_whole<T>(p, i + 16 * (x0 + x), j, g, u);
                }
                continue;
            }
#pragma unroll 1
            for (int at = 0; at < kN; ++at) {
                const int x = at / (kN / 4), y = at % (kN / 4) * 2;
                float g[8], u[8];
                fetch(x, y, g, u);
                Kind::template put<T>(p, t.part, i + 16 * (x0 + x), j + 16 * y, g, u);
            }
        }
        return;
    } else {
    // A wave passes its sums through a place of the ring of its own, 64 rows at a time, so
    // that a lane gets eight neighbouring columns; no barrier of the workgroup is needed, the
    // fences keep the lanes' writes before other lanes' reads, and those before the next writes.
    constexpr int kWide = kTile / 2, kTurnRows = 64;
    static_assert(kTurnRows * kWide * 4 <= kBytes && kWide % kTurnRows == 0);
    float* const turn = reinterpret_cast<float*>(wave == 0 ? r0 : wave == 1 ? r1 : wave == 2 ? r2 : r3);
    const auto place = [](int row, int column) { return row * kWide + (column ^ row / 4 % 4 * 16); };
    Kind::template finish<T, kWide>(p, t.part, turn, place, i0 + wi, j0 + wj, [&](auto each) {
#pragma unroll
        for (int x0 = 0; x0 < kN; x0 += 4) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < kN; ++y)
#pragma unroll
                    for (int r = 0; r < 4; ++r) turn[place(16 * x + 4 * (lane / 16) + r, 16 * y + lane % 16)] = acc[x0 + x][y][r];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            each(16 * x0, kTurnRows);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    });
    }
}

}  // namespace
}  // namespace fsdp_block
