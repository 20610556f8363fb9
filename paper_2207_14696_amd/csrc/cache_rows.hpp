// What the kernels that write and read rows of the paged cache share: rows of head_dim columns, each with a range of its own.
#pragma once

#include <type_traits>

#include "cache.hpp"

namespace bf {
namespace {

// A workgroup takes up to kTokens tokens of the call, all their heads, keys and values.  Where they lie in the cache is looked up
// once a token.  Then LPR lanes take a row, 8 columns each; a wave's rows are consecutive tokens' of a head, which lie next to
// each other in a page as far as the call's tokens do in their sequence.
constexpr int kTokens = 16;

struct Places {
    int64_t page[kTokens];  // byte offset of the page, -1: before the sequence's beginning
    int slot[kTokens];
    int position[kTokens];  // in the sequence
};

__device__ inline void find_places(const CachePages &c, const CacheBatch &b, int64_t t0, int count, Places &sh) {
    if (threadIdx.x < 64) {
        int seq = sequence_of(b, t0);
        if ((int)threadIdx.x < count) {
            const int64_t t = t0 + threadIdx.x;
            if (b.indptr)
                while (seq + 1 < b.B && b.indptr[seq + 1] <= t) seq++;
            else
                seq = (int)(t / b.n);
            const int64_t pos = b.length(seq, c.ps_log2) - b.count(seq) + (t - b.first(seq));
            sh.slot[threadIdx.x] = (int)(pos & (c.ps() - 1));
            sh.position[threadIdx.x] = (int)pos;
            sh.page[threadIdx.x] = pos < 0 ? -1 : b.tables[(int64_t)seq * b.width + (pos >> c.ps_log2)] * c.page_bytes;
        }
    }
    __syncthreads();
}

// the smallest, or largest, of LPR neighbouring lanes' values, in all of them
template <int LPR, bool MAX>
__device__ inline float extreme(float x) {
    auto of = [](float a, float b) { return MAX ? fmaxf(a, b) : fminf(a, b); };
    auto moved = [](float a, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, a), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    x = of(x, moved(x, std::integral_constant<int, 0xb1>{}));   // lane ^ 1
    x = of(x, moved(x, std::integral_constant<int, 0x4e>{}));   // lane ^ 2
    x = of(x, moved(x, std::integral_constant<int, 0x141>{}));  // the other four of eight
    if constexpr (LPR > 8) x = of(x, moved(x, std::integral_constant<int, 0x140>{}));  // the other eight of sixteen
    if constexpr (LPR > 16) x = of(x, __shfl_xor(x, 16));
    return x;
}

// Eight of a row's columns by each of its LPR lanes.  All lanes of a wave.
template <int BITS, int LPR>
__device__ inline void write_row(const CachePages &c, const float (&x)[8], bool real, uint8_t *block, int which, int slot) {
    const int sub = threadIdx.x % LPR, col = 8 * sub;
    float mn = INFINITY, mx = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (col + i < c.d) {
            nan |= x[i] != x[i];
            mn = fminf(mn, x[i]);
            mx = fmaxf(mx, x[i]);
        }
    const uint64_t nans = __ballot(nan) >> (threadIdx.x % 64 / LPR * LPR);
    const bool any_nan = (uint32_t)nans & (uint32_t)((1ull << LPR) - 1);
    mn = extreme<LPR, false>(mn);
    mx = extreme<LPR, true>(mx);
    if (!real) return;
    constexpr float kTop = (1 << BITS) - 1;
    const float span = mx - mn;
    float inv = kTop / span, scale = span / kTop;
    if (!(fabsf(inv) <= 3.402823466e38f)) inv = scale = 0.f;
    if (any_nan || !(span <= 3.402823466e38f)) {  // (an infinity makes the span infinite or NaN)
        mn = scale = NAN;
        inv = 0.f;
    }
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float f = fminf(fmaxf(rintf((x[i] - mn) * inv), 0.f), kTop);  // (a NaN becomes 0)
        q[i] = col + i < c.d ? (uint32_t)f : 0u;
    }
    uint8_t *codes = block + c.codes(which) + slot * c.rb;
    if (sub * BITS < c.rb) {  // 8 codes are BITS bytes
        if constexpr (BITS == 8) {
            uint2 w;
            w.x = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
            w.y = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
            *reinterpret_cast<uint2 *>(codes + 8 * sub) = w;
        } else {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) w |= q[i] << 4 * i;
            *reinterpret_cast<uint32_t *>(codes + 4 * sub) = w;
        }
    }
    if (sub == 0) {
        float *f = reinterpret_cast<float *>(block + c.floats(which)) + slot;
        f[0] = scale;
        f[c.ps()] = mn;
    }
}

inline int lanes_per_row(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

}  // namespace
}  // namespace bf
