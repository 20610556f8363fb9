// The paged cache written and read back: rows of head_dim columns, each with a range of its own.
#include <algorithm>
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

// Bound by the bytes of k and v and of the codes: 65 536 tokens of 8 heads of 128, bf16 to 8 bits (268 MB read, 143 written) 112 us,
// 3.7 TB/s; fp32 (537 MB read) 153, 4.4 TB/s.  A row's codes are 128 bytes of a page, its two floats 8 more, elsewhere in it.
template <typename T, int BITS, int LPR>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CachePages c, CacheBatch b, HeadRows k, HeadRows v, int per) {
    __shared__ Places places;
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const int count = b.tokens - t0 < per ? (int)(b.tokens - t0) : per;
    find_places(c, b, t0, count, places);
    const int sub = threadIdx.x % LPR, col = 8 * sub, rows = count * 2 * c.heads;
    // (a wave's rows are taken together, those past the end as zeros that are not stored; a row at a time: with two on their way
    // fewer waves fit, and 65 536 tokens took 121 us where they now take 112)
    for (int r0 = threadIdx.x / 64 * (64 / LPR); r0 < rows; r0 += kThreads / LPR) {
        const int r = r0 + threadIdx.x % 64 / LPR, token = r % count, hw = r / count, which = hw >= c.heads, head = hw - which * c.heads;
        const bool real = r < rows && places.page[token] >= 0;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = 0.f;
        if (real) {
            const HeadRows &h = which ? v : k;
            load8_any(static_cast<const T *>(h.data) + (t0 + token) * h.token_stride + head * h.head_stride + col, c.d - col, x);
        }
        write_row<BITS, LPR>(c, x, real, c.pages + places.page[token] + head * c.head_bytes, which, places.slot[token]);
    }
}

// Bound by the bytes of the result, twice (fp32: four times) the codes'.  STREAMED past the caches from 16 MB on:
// 149 000 tokens of 8 heads of 128 in 8 bits to bf16 (610 MB written, 320 read) 257 us, 167 so (5.6 TB/s); 32 MB 10.5 us, 8.7 so; 256 MB 81.5 and
// 63.  A program that goes through the result next gives some of that back: with k and v scaled in place after it, 32 MB 26.3 us, 28.3 so;
// 256 MB 154 and 161.
// 65 536 tokens to fp32 (537 MB written) 143 us, 104 so; with a lane's eight columns next to each other, half a line a store, 257.
template <typename T, int BITS, int LPR, bool STREAMED>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CachePages c, CacheBatch b, T *k, T *v, int per) {
    __shared__ Places places;
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const int count = b.tokens - t0 < per ? (int)(b.tokens - t0) : per;
    find_places(c, b, t0, count, places);
    // a lane's columns: eight next to each other, in fp32 four and four, so that each store of a row's lanes fills whole lines
    constexpr int kSets = sizeof(T) == 4 ? 2 : 1, kCols = 8 / kSets, kBytes = kCols * BITS / 8, kWords = (kBytes + 3) / 4;
    const int sub = threadIdx.x % LPR, col = kCols * sub, rows = count * 2 * c.heads;
    if (col >= c.d) return;
    constexpr int kAhead = 8;  // rows in flight
    for (int r0 = threadIdx.x / LPR; r0 < rows; r0 += kAhead * (kThreads / LPR)) {
        uint32_t w[kAhead][kSets][kWords];
        float scale[kAhead], mn[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int r = r0 + i * (kThreads / LPR), token = r % count, hw = r / count, which = hw >= c.heads, head = hw - which * c.heads;
            scale[i] = mn[i] = 0.f;
#pragma unroll
            for (int g = 0; g < kSets; g++)
#pragma unroll
                for (int e = 0; e < kWords; e++) w[i][g][e] = 0;
            if (r < rows && places.page[token] >= 0) {
                const uint8_t *block = c.pages + places.page[token] + head * c.head_bytes;
                const int slot = places.slot[token];
                const uint8_t *codes = block + c.codes(which) + slot * c.rb;
#pragma unroll
                for (int g = 0; g < kSets; g++)
                    if (g == 0 || col + g * kCols * LPR < c.d)
                        __builtin_memcpy(w[i][g], __builtin_assume_aligned(codes + kBytes * (sub + g * LPR), kBytes), kBytes);
                const float *f = reinterpret_cast<const float *>(block + c.floats(which)) + slot;
                scale[i] = f[0], mn[i] = f[c.ps()];
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int r = r0 + i * (kThreads / LPR), token = r % count, hw = r / count, which = hw >= c.heads, head = hw - which * c.heads;
            if (r >= rows) break;
            T *row = (which ? v : k) + ((t0 + token) * c.heads + head) * c.d;
#pragma unroll
            for (int g = 0; g < kSets; g++) {
                float x[kCols];
#pragma unroll
                for (int e = 0; e < kCols; e++) {
                    const uint32_t q = w[i][g][e * BITS / 32] >> e * BITS % 32 & ((1u << BITS) - 1);
                    x[e] = fmaf((float)q, scale[i], mn[i]);
                }
                const int at = col + g * kCols * LPR;
                if (g == 0 || at < c.d) store_any<kCols, STREAMED>(row + at, c.d - at, x);
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void cache_check_kernel(CacheBatch b, int ps_log2, int64_t num_pages, int32_t *bad) {
    int wrong = 0;
    const int64_t stride = (int64_t)gridDim.x * kThreads, me = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    for (int64_t i = me; i < (int64_t)b.B * b.width; i += stride) {
        const int64_t seq = i / b.width, page = i - seq * b.width;
        if (page << ps_log2 < b.lengths[seq]) wrong |= b.tables[i] < 0 || b.tables[i] >= num_pages;
    }
    for (int64_t i = me; i < b.B; i += stride) {
        wrong |= b.lengths[i] < 0 || b.lengths[i] > b.width << ps_log2;
        if (b.indptr) wrong |= b.indptr[i] > b.indptr[i + 1] || b.indptr[i] < 0;
    }
    if (me == 0 && b.indptr) wrong |= b.indptr[0] != 0 || b.indptr[b.B] != b.tokens;
    if (wrong) atomicOr(bad, 1);
}

__global__ void cache_check_zero_kernel(int32_t *bad) { *bad = 0; }

int lanes_per_row(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

// Tokens a workgroup: up to 16, whose places are looked up at once, where that leaves so many workgroups.  8 heads of 128 in 8 bits, bf16:
// written with 2048 8192 tokens take 17.7 us, 32 768 56 (with 8192: 20.5 and 53); read with 1024 4096 take 6.0 (with 2048: 9.3),
// 8192 to fp32 14.3 (with 512: 16.3).
int tokens_per(const CacheBatch &b, int workgroups) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(kTokens, b.tokens / workgroups));
}
unsigned row_blocks(const CacheBatch &b, int per) { return (unsigned)((b.tokens + per - 1) / per); }

}  // namespace

#define BF_BY_TYPE(CALL)                              \
    if (dtype == BIFEAT_F32) { CALL(float); }         \
    else if (dtype == BIFEAT_F16) { CALL(Half16); }   \
    else { CALL(Brain16); }

hipError_t launch_cache_write(const CachePages &c, const CacheBatch &b, const HeadRows &k, const HeadRows &v, int bits, int dtype,
                              hipStream_t s) {
    const int lpr = lanes_per_row(c.d), per = tokens_per(b, 2048);
    const unsigned grid = row_blocks(b, per);
#define BF_GO(T, LPR)                                                                     \
    if (bits == 8) cache_write_kernel<T, 8, LPR><<<grid, kThreads, 0, s>>>(c, b, k, v, per);   \
    else cache_write_kernel<T, 4, LPR><<<grid, kThreads, 0, s>>>(c, b, k, v, per)
#define BF_LPR(T) if (lpr == 8) { BF_GO(T, 8); } else if (lpr == 16) { BF_GO(T, 16); } else { BF_GO(T, 32); }
    BF_BY_TYPE(BF_LPR)
#undef BF_GO
    return hipGetLastError();
}

hipError_t launch_cache_read(const CachePages &c, const CacheBatch &b, void *k, void *v, int bits, int dtype, hipStream_t s) {
    const int lpr = lanes_per_row(c.d), per = tokens_per(b, 1024);
    const unsigned grid = row_blocks(b, per);
    const bool stream = b.tokens * 2 * c.heads * c.d * (dtype == BIFEAT_F32 ? 4 : 2) > (16 << 20);
#define BF_GO(T, LPR)                                                                                                             \
    if (bits == 8) {                                                                                                              \
        if (stream) cache_read_kernel<T, 8, LPR, true><<<grid, kThreads, 0, s>>>(c, b, (T *)k, (T *)v, per);                      \
        else cache_read_kernel<T, 8, LPR, false><<<grid, kThreads, 0, s>>>(c, b, (T *)k, (T *)v, per);                            \
    } else {                                                                                                                      \
        if (stream) cache_read_kernel<T, 4, LPR, true><<<grid, kThreads, 0, s>>>(c, b, (T *)k, (T *)v, per);                      \
        else cache_read_kernel<T, 4, LPR, false><<<grid, kThreads, 0, s>>>(c, b, (T *)k, (T *)v, per);                            \
    }
    BF_BY_TYPE(BF_LPR)
#undef BF_GO
#undef BF_LPR
    return hipGetLastError();
}

void launch_cache_check(const CacheBatch &b, int ps_log2, int64_t num_pages, int32_t *d_bad, hipStream_t s) {
    cache_check_zero_kernel<<<1, 1, 0, s>>>(d_bad);
    cache_check_kernel<<<blocks_for(std::max<int64_t>(b.B * b.width, 1)), kThreads, 0, s>>>(b, ps_log2, num_pages, d_bad);
}

}  // namespace bf
