#pragma once

#include "cache_attend_chunk_impl.hpp"

namespace bf {

template <int BITS, int DP, int NP>
hipError_t attend_chunk_one(const AttendCall &a, const AttendPlan &p) {
    constexpr int kNT = chunk_tiles(DP, NP);
    constexpr size_t lds = chunk_lds<BITS, DP, kNT>();
    const int mode = mode_of(a);
    auto kernel = mode == kCapped  ? attend_chunk_kernel<BITS, DP, NP, kNT, kCapped>
                  : mode == kBiased ? attend_chunk_kernel<BITS, DP, NP, kNT, kBiased>
                                    : attend_chunk_kernel<BITS, DP, NP, kNT, kPlain>;
    if constexpr (NP == 1)
        if (mode == kCappedFirst) kernel = attend_chunk_kernel<BITS, DP, NP, kNT, kCappedFirst>;
    if (lds > 64 * 1024) {  // (what a launch may have without being asked)
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) return e;
    }
    kernel<<<grid_of(p), 256, lds, a.s>>>(a, p);
    return hipSuccess;
}

template <int BITS>
hipError_t attend_chunk_bits(const AttendCall &a, const AttendPlan &p, int dp) {
    const bool wide = a.dtype == BIFEAT_F32;
    if (dp == 64) return wide ? attend_chunk_one<BITS, 64, 2>(a, p) : attend_chunk_one<BITS, 64, 1>(a, p);
    if (dp == 128) return wide ? attend_chunk_one<BITS, 128, 2>(a, p) : attend_chunk_one<BITS, 128, 1>(a, p);
    return wide ? attend_chunk_one<BITS, 256, 2>(a, p) : attend_chunk_one<BITS, 256, 1>(a, p);
}

}  // namespace bf
