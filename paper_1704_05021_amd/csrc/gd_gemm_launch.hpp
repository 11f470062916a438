// Picks the tile and the split of k of a product, and launches it.
#pragma once

#include "gd_gemm.hpp"

namespace gd {

constexpr uint64_t kUnits = 256;  // compute units

// Multiplications from which padded copies of ragged operands pay: the copies cost two launches, the form without them
// passes operands through registers and transposes there those across k.  Forward 2001 x 2001 x 2001 takes 33 us without
// and 45 with them, 3001 x 3001 x 1501 70 and 57; the input's gradient of those 40 and 44, 68 and 46; the weight's
// gradient of 1000 x 1001 x 1001 18 and 17, of 8000 x 301 x 999 39 and 33.
constexpr double pad_work(int form) { return form == kAlong ? 1e10 : form == kPAcross ? 7e9 : 1e9; }

// Whether rows of an operand start at 16-byte boundaries and are whole 16-byte chunks long.
template <typename E>
bool whole_chunks(const void* p, uint64_t stride, uint64_t columns) {
    constexpr uint32_t CE = 16 / sizeof(E);
    return ((uintptr_t)p & 15) == 0 && stride % CE == 0 && columns % CE == 0;
}

// Puts a padded copy of [rows][columns] in place of p, where there is room.
template <typename E>
bool pad(const void*& p, uint64_t& stride, uint64_t rows, uint32_t columns, GemmRoom& room, hipStream_t st) {
    constexpr uint32_t CE = 16 / sizeof(E);
    const uint64_t per_row = (columns + CE - 1) / CE, bytes = rows * per_row * 16;
    if (bytes > room.pad_bytes) return false;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((rows * per_row + kBlock - 1) / kBlock, 1u << 16);
    k_pad<E><<<dim3(blocks), dim3(kBlock), 0, st>>>((const E*)p, stride, rows, columns, (E*)room.pad);
    p = room.pad;
    stride = per_row * CE;
    room.pad += bytes;
    room.pad_bytes -= bytes;
    return true;
}

// What a tile costs, in microseconds, measured on products in bfloat16 with k
// of 4,096 (64 steps): a step of one tile alone on its compute unit, and of
// each of several there at once (as many as LDS holds).  Every round of tiles
// also takes about kRoundUs to fill the pipeline and write results.  Products
// in binary32, of 8 bits and through registers are planned with the same
// figures, which are not theirs: their steps take longer (binary32 about four
// times as long: 8192 x 4096 x 4096 is planned at 506 us and takes 1,970; through
// registers in bfloat16 it takes 346), so the split of k and the join weigh
// more in their plans than they should.
struct TileCost {
    uint32_t bi, bj, threads, at_once;
    double alone_us, shared_us;
    uint64_t tiles(uint64_t I, uint64_t J) const { return ((I + bi - 1) / bi) * ((J + bj - 1) / bj); }
    bool fits(uint64_t I, uint64_t J) const { return tiles(I, J) * threads <= 0xFFFFFFFFull; }  // threads of a dispatch
};
constexpr TileCost kBigCost{256, 256, TileBig::kThreads, 1, 1.48, 1.48}, kLongCost{256, 192, TileLong::kThreads, 1, 1.10, 1.10},
    kWideCost{256, 128, TileWide::kThreads, 1, 0.82, 0.82}, kMidCost{128, 128, TileMid::kThreads, 2, 0.58, 0.475},
    kSmallCost{64, 64, TileSmall::kThreads, 2, 0.17, 0.165};
static_assert(TileMid::BI == kProductTile && TileMid::BJ == kProductTile && TileMid::kThreads == kProductThreads,
              "the tile that every product which product_fits can take");
constexpr double kRoundUs = 5.0, kJoinUs = 4.0, kJoinBytesPerUs = 3.5e6;

struct TilePlan {
    double us;
    uint32_t splits;
};

// The number of shares of k that a product of `steps` steps does best with, and its time: shares fill compute units
// that the tiles leave idle, and cost the writing and reading of their sums.
inline TilePlan plan_tiles(const TileCost& c, uint64_t I, uint64_t J, uint64_t steps, uint64_t room) {
    const uint64_t tiles = c.tiles(I, J);
    const auto time = [&](uint64_t splits) {
        const uint64_t each = (steps + splits - 1) / splits, load = (tiles * splits + kUnits - 1) / kUnits;
        const auto round = [&](uint64_t n) {
            return n ? (double)each * std::max(c.alone_us, (double)n * c.shared_us) + kRoundUs : 0.0;
        };
        const double join = splits > 1 ? kJoinUs + 8.0 * (double)(splits * I) * (double)J / kJoinBytesPerUs : 0.0;
        return (double)(load / c.at_once) * round(c.at_once) + round(load % c.at_once) + join;
    };
    TilePlan best{time(1), 1};
    for (uint64_t s = 2; s <= 64 && s * 4 <= steps && s * I * J <= room; s += s < 4 ? 1 : s / 4 * 2) {
        const double us = time(s);
        if (us < best.us) best = {us, (uint32_t)s};
    }
    return best;
}

template <typename E, typename O, int FORM, typename TL, bool PAIR = false>
hipError_t launch_tiles(GemmArgs a, uint64_t splits, bool direct, hipStream_t st) {
    constexpr uint32_t KE = kStepBytes / sizeof(E), kResults = PAIR ? TL::BI / 2 : TL::BI;
    a.tiles_i = (a.I + kResults - 1) / kResults;
    a.tiles_j = (a.J + TL::BJ - 1) / TL::BJ;
    const uint64_t tiles = (uint64_t)a.tiles_i * a.tiles_j, steps = ((uint64_t)a.K + KE - 1) / KE;
    a.steps = (uint32_t)((steps + splits - 1) / splits);
    if (a.steps) splits = (steps + a.steps - 1) / a.steps;
    float* part = a.part;
    if (splits == 1) a.part = nullptr;
    const dim3 grid((uint32_t)tiles, (uint32_t)splits);
    if constexpr (sizeof(E) <= 2) {
        if (direct) k_gemm_fetch<E, O, FORM >= kPAcross, FORM == kBothAcross, TL, PAIR><<<grid, dim3(TL::kThreads), 0, st>>>(a);
    }
    if constexpr (TL::kThreads <= kBlock) {
        if (!direct) k_gemm<E, O, FORM >= kPAcross, FORM == kBothAcross, TL, PAIR><<<grid, dim3(TL::kThreads), 0, st>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    a.part = part;
    const uint64_t threads = (uint64_t)((a.I + 3) / 4) * a.J;
    k_join<E, O, PAIR><<<dim3((uint32_t)std::min<uint64_t>((threads + kBlock - 1) / kBlock, 1u << 16)), dim3(kBlock), 0, st>>>(
        a, (uint32_t)splits);
    return hipGetLastError();
}

// The tile (0 the smallest) and the split of k of a product with I rows of P.
struct Choice {
    int tile;
    uint32_t splits;
};
template <typename E, int FORM>
Choice choose(const GemmArgs& a, uint64_t I, bool direct, uint64_t room) {
    constexpr uint32_t KE = kStepBytes / sizeof(E);
    const uint64_t steps = ((uint64_t)a.K + KE - 1) / KE;
    TilePlan best{1e300, 1};
    int tile = 0;
    constexpr TileCost kCosts[] = {kSmallCost, kMidCost, kWideCost, kLongCost, kBigCost};
    for (int t = 0; t < (direct ? 5 : 2); ++t) {  // the larger tiles take operands placed in LDS only
        if (FORM == kBothAcross && t == 3) continue;  // rows of 192 across k would not be a power of two in LDS
        if (!kCosts[t].fits(I, a.J)) continue;
        const TilePlan p = plan_tiles(kCosts[t], I, a.J, steps, room);
        if (p.us < best.us) best = p, tile = t;
    }
    return {tile, best.splits};
}

template <typename E, typename O, int FORM, bool PAIR>
hipError_t launch_product(GemmArgs a, const GemmRoom& given, hipStream_t st) {
    static_assert(!PAIR || FORM == kAlong);
    const uint32_t rows_of_p = PAIR ? 2 * a.I : a.I;
    if constexpr (FORM == kAlong)
        if (a.J <= (uint32_t)kThinRows) {
            k_thin<E, O, PAIR><<<dim3((a.I + kThinRows - 1) / kThinRows), dim3(kThinWaves * kWave), 0, st>>>(a);
            return hipGetLastError();
        }
    // 32 MB is what the dies' L2 hold together (8192 x 4096 x 4096 in bfloat16: 197 us stored past them, 213 through)
    a.fin.stream = (uint64_t)a.I * a.J * sizeof(O) >= 32ull << 20;
    bool direct = false;
    if constexpr (sizeof(E) <= 2) {
        const uint64_t p_rows = FORM >= kPAcross ? a.K : rows_of_p, q_rows = FORM == kBothAcross ? a.K : a.J;
        const uint32_t p_cols = FORM >= kPAcross ? a.I : a.K, q_cols = FORM == kBothAcross ? a.J : a.K;
        const bool p_whole = whole_chunks<E>(a.p, a.p_stride, p_cols), q_whole = whole_chunks<E>(a.q, a.q_stride, q_cols);
        direct = p_whole && q_whole;
        GemmRoom room = given;
        if (!direct && room.pad && a.K && (double)rows_of_p * a.J * a.K >= pad_work(FORM)) {
            GemmArgs b = a;
            direct = (p_whole || pad<E>(b.p, b.p_stride, p_rows, p_cols, room, st)) &&
                     (q_whole || pad<E>(b.q, b.q_stride, q_rows, q_cols, room, st));
            if (direct) a = b;
        }
    }
    const Choice best = choose<E, FORM>(a, rows_of_p, direct, given.floats);
    const auto run = [&](auto tl) { return launch_tiles<E, O, FORM, decltype(tl), PAIR>(a, best.splits, direct, st); };
    const int tile = best.tile;
    if constexpr (sizeof(E) <= 2) {
        if (tile == 4) return run(TileBig());
        if constexpr (FORM != kBothAcross)
            if (tile == 3) return run(TileLong());
        if (tile == 2) return run(TileWide());
    }
    return tile == 1 ? run(TileMid()) : run(TileSmall());
}

template <typename E, typename O, int FORM>
hipError_t launch_gemm(GemmArgs a, const GemmRoom& room, hipStream_t st) {
    return launch_product<E, O, FORM, false>(a, room, st);
}
template <typename E, typename O>
hipError_t launch_gated(const GemmArgs& a, const GemmRoom& room, hipStream_t st) {
    return launch_product<E, O, kAlong, true>(a, room, st);
}

// Both products in one launch, where each takes the smallest tile and does
// not split k (40 x 784 x 512: 11.6 us in place of 15.0).
template <typename T>
bool pair_backward(GemmArgs dx, GemmArgs dw, const GemmRoom& room, hipStream_t st, hipError_t& e) {
    const bool direct = sizeof(T) == 2 && whole_chunks<T>(dx.p, dx.p_stride, dx.I) &&
                        whole_chunks<T>(dx.q, dx.q_stride, dx.K) && whole_chunks<T>(dw.p, dw.p_stride, dw.I);
    if (!direct && room.pad && (double)dx.I * dx.J * dx.K >= pad_work(kBothAcross)) return false;
    const Choice a = choose<T, kPAcross>(dx, dx.I, direct, room.floats), b = choose<T, kBothAcross>(dw, dw.I, direct, room.floats);
    if (a.tile || b.tile || a.splits > 1 || b.splits > 1) return false;
    uint64_t blocks = 0, first = 0;
    for (GemmArgs* g : {&dx, &dw}) {
        constexpr uint32_t KE = kStepBytes / sizeof(T);
        g->tiles_i = (g->I + TileSmall::BI - 1) / TileSmall::BI;
        g->tiles_j = (g->J + TileSmall::BJ - 1) / TileSmall::BJ;
        g->steps = (g->K + KE - 1) / KE;
        g->part = nullptr;
        first = blocks;
        blocks += (uint64_t)g->tiles_i * g->tiles_j;
    }
    if (blocks * TileSmall::kThreads > 0xFFFFFFFFull) return false;
    const dim3 grid((uint32_t)blocks), block(TileSmall::kThreads);
    if constexpr (sizeof(T) == 2)
        if (direct) k_gemm_pair<T, true><<<grid, block, 0, st>>>(dx, dw, (uint32_t)first);
    if (!direct) k_gemm_pair<T, false><<<grid, block, 0, st>>>(dx, dw, (uint32_t)first);
    e = hipGetLastError();
    return true;
}

template <typename T>
hipError_t launch_backward(const GemmArgs* dx, const GemmArgs* dw, const GemmRoom& room, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (dx && dw && pair_backward<T>(*dx, *dw, room, st, e)) return e;
    if (dx) e = launch_gemm<T, T, kPAcross>(*dx, room, st);
    if (dw && e == hipSuccess) e = launch_gemm<T, float, kBothAcross>(*dw, room, st);
    return e;
}

}  // namespace gd
