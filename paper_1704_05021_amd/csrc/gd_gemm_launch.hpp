// Picks the tile and the split of k of a product, and launches it.
#pragma once

#include "gd_gemm.hpp"

namespace gd {

// Whether every row of both operands starts and ends at a 16-byte boundary.
template <typename E, int FORM>
bool whole_chunks(const GemmArgs& a) {
    constexpr uint32_t CE = 16 / sizeof(E);
    if (sizeof(E) > 2) return false;
    const bool aligned = (((uintptr_t)a.p | (uintptr_t)a.q) & 15) == 0 && a.p_stride % CE == 0 && a.q_stride % CE == 0;
    return aligned && (FORM == kBothAcross || a.K % CE == 0) && (FORM == kAlong || a.I % CE == 0) &&
           (FORM != kBothAcross || a.J % CE == 0);
}

template <typename E, typename O, int FORM, typename TL>
hipError_t launch_tiles(GemmArgs a, uint64_t room, hipStream_t st) {
    const bool direct = whole_chunks<E, FORM>(a);
    const uint32_t KE = (direct ? kLineBytes : kStepBytes) / sizeof(E);
    a.tiles_i = (a.I + TL::BI - 1) / TL::BI;
    a.tiles_j = (a.J + TL::BJ - 1) / TL::BJ;
    const uint64_t tiles = (uint64_t)a.tiles_i * a.tiles_j, steps = ((uint64_t)a.K + KE - 1) / KE;
    if (tiles * TL::kThreads > 0xFFFFFFFFull) return hipErrorInvalidValue;
    // k is split where the tiles leave most of the 256 compute units idle, into shares of at least four steps
    uint64_t splits = 1;
    if (tiles < 256) {
        splits = std::min<uint64_t>(512 / tiles, steps / 4);
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
    if (!direct) k_gemm<E, O, FORM >= kPAcross, FORM == kBothAcross, TL><<<grid, dim3(TL::kThreads), 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    a.part = part;
    const uint64_t threads = (uint64_t)((a.I + 3) / 4) * a.J;
    k_join<E, O><<<dim3((uint32_t)std::min<uint64_t>((threads + kBlock - 1) / kBlock, 1u << 16)), dim3(kBlock), 0, st>>>(
        a, (uint32_t)splits);
    return hipGetLastError();
}

template <typename E, typename O, int FORM>
hipError_t launch_gemm(GemmArgs a, uint64_t room, hipStream_t st) {
    if constexpr (FORM == kAlong)
        if (a.J <= (uint32_t)kThinRows) {
            k_thin<E, O><<<dim3((a.I + kThinRows - 1) / kThinRows), dim3(kThinWaves * kWave), 0, st>>>(a);
            return hipGetLastError();
        }
    const auto tiles = [&](uint64_t b) { return ((a.I + b - 1) / b) * ((a.J + b - 1) / b); };
    if (tiles(256) >= 200) return launch_tiles<E, O, FORM, TileBig>(a, room, st);
    if (tiles(128) >= 200) return launch_tiles<E, O, FORM, TileMid>(a, room, st);
    return launch_tiles<E, O, FORM, TileSmall>(a, room, st);
}

}  // namespace gd
