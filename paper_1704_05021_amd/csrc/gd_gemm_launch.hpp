// Picks the tile and the split of k of a product, and launches it.
#pragma once

#include "gd_gemm.hpp"

namespace gd {

constexpr uint64_t kUnits = 256;  // compute units
constexpr double kPadWork = 2e8;  // products from which padded copies pay

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

template <typename E, typename O, int FORM, typename TL>
hipError_t launch_tiles(GemmArgs a, uint64_t room, bool direct, hipStream_t st) {
    constexpr uint32_t KE = kStepBytes / sizeof(E);
    a.tiles_i = (a.I + TL::BI - 1) / TL::BI;
    a.tiles_j = (a.J + TL::BJ - 1) / TL::BJ;
    const uint64_t tiles = (uint64_t)a.tiles_i * a.tiles_j, steps = ((uint64_t)a.K + KE - 1) / KE;
    if (tiles * TL::kThreads > 0xFFFFFFFFull) return hipErrorInvalidValue;
    // k is split where the tiles leave most of the compute units idle, into shares of at least four steps
    uint64_t splits = 1;
    if (tiles < kUnits) {
        splits = std::min<uint64_t>(2 * kUnits / tiles, steps / 4);
        splits = std::min<uint64_t>(splits, room / ((uint64_t)a.I * a.J));
        splits = std::max<uint64_t>(splits, 1);
    }
    a.steps = (uint32_t)((steps + splits - 1) / splits);
    if (a.steps) splits = (steps + a.steps - 1) / a.steps;
    float* part = a.part;
    if (splits == 1) a.part = nullptr;
    const dim3 grid((uint32_t)tiles, (uint32_t)splits);
    if constexpr (sizeof(E) <= 2) {
        if (direct) k_gemm_fetch<E, O, FORM >= kPAcross, FORM == kBothAcross, TL><<<grid, dim3(TL::kThreads), 0, st>>>(a);
    }
    if constexpr (TL::kThreads <= kBlock) {
        if (!direct) k_gemm<E, O, FORM >= kPAcross, FORM == kBothAcross, TL><<<grid, dim3(TL::kThreads), 0, st>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    a.part = part;
    const uint64_t threads = (uint64_t)((a.I + 3) / 4) * a.J;
    k_join<E, O><<<dim3((uint32_t)std::min<uint64_t>((threads + kBlock - 1) / kBlock, 1u << 16)), dim3(kBlock), 0, st>>>(
        a, (uint32_t)splits);
    return hipGetLastError();
}

template <typename E, typename O, int FORM>
hipError_t launch_gemm(GemmArgs a, const GemmRoom& given, hipStream_t st) {
    if constexpr (FORM == kAlong)
        if (a.J <= (uint32_t)kThinRows) {
            k_thin<E, O><<<dim3((a.I + kThinRows - 1) / kThinRows), dim3(kThinWaves * kWave), 0, st>>>(a);
            return hipGetLastError();
        }
    bool direct = false;
    if constexpr (sizeof(E) <= 2) {
        const uint64_t p_rows = FORM >= kPAcross ? a.K : a.I, q_rows = FORM == kBothAcross ? a.K : a.J;
        const uint32_t p_cols = FORM >= kPAcross ? a.I : a.K, q_cols = FORM == kBothAcross ? a.J : a.K;
        const bool p_whole = whole_chunks<E>(a.p, a.p_stride, p_cols), q_whole = whole_chunks<E>(a.q, a.q_stride, q_cols);
        direct = p_whole && q_whole;
        GemmRoom room = given;
        if (!direct && room.pad && a.K && (double)a.I * a.J * a.K >= kPadWork) {
            GemmArgs b = a;
            direct = (p_whole || pad<E>(b.p, b.p_stride, p_rows, p_cols, room, st)) &&
                     (q_whole || pad<E>(b.q, b.q_stride, q_rows, q_cols, room, st));
            if (direct) a = b;
        }
    }
    const auto tiles = [&](uint64_t b) { return ((a.I + b - 1) / b) * ((a.J + b - 1) / b); };
    const uint64_t room = given.floats;
    if constexpr (sizeof(E) <= 2)
        if (direct && tiles(256) >= 200) return launch_tiles<E, O, FORM, TileBig>(a, room, direct, st);
    if (tiles(128) >= 200) return launch_tiles<E, O, FORM, TileMid>(a, room, direct, st);
    return launch_tiles<E, O, FORM, TileSmall>(a, room, direct, st);
}

}  // namespace gd
