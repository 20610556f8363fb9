// The paged cache written and read back: rows of head_dim columns, each with a range of its own.
#include <algorithm>

#include "cache.hpp"

namespace bf {
namespace {

// LPR lanes a row, 8 columns a lane; rows of a token are its heads' keys, then its heads' values, so that a
// wave's rows are a few tokens'.  The place of a wave's first token is looked up by the whole wave.
struct RowPlace {
    bool there;     // a row of the call, with a place in the cache
    int64_t token;  // of the call
    int which, head;
    int64_t slot;
    uint8_t *block;
};

template <int LPR>
__device__ inline RowPlace place_row(const CachePages &c, const CacheBatch &b, int64_t &row, bool &in_call) {
    const int64_t wave = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const int64_t first_row = wave * (64 / LPR);
    const int per = 2 * c.heads;
    int64_t t0 = first_row / per;
    if (t0 >= b.tokens) t0 = b.tokens - 1;
    int seq = sequence_of(b, t0);
    row = first_row + (threadIdx.x & 63) / LPR;
    RowPlace p;
    p.token = row / per;
    in_call = p.token < b.tokens;
    const int r = (int)(row - p.token * per);
    p.which = r >= c.heads;
    p.head = r - p.which * c.heads;
    p.there = false;
    p.slot = 0;
    p.block = nullptr;
    if (!in_call) return p;
    if (b.indptr)
        while (seq + 1 < b.B && b.indptr[seq + 1] <= p.token) seq++;
    else
        seq = (int)(p.token / b.n);
    const int64_t pos = b.length(seq, c.ps_log2) - b.count(seq) + (p.token - b.first(seq));
    if (pos < 0) return p;
    p.there = true;
    p.slot = pos & (c.ps() - 1);
    p.block = c.block(b.tables[(int64_t)seq * b.width + (pos >> c.ps_log2)], p.head);
    return p;
}

template <typename T, int BITS, int LPR>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(CachePages c, CacheBatch b, HeadRows k, HeadRows v) {
    int64_t row;
    bool in_call;
    const RowPlace p = place_row<LPR>(c, b, row, in_call);
    const int sub = threadIdx.x % LPR, col = 8 * sub;
    float x[8];
    float mn = INFINITY, mx = -INFINITY;
    int bad = 0;
    if (p.there) {
        const HeadRows &h = p.which ? v : k;
        load8_any(static_cast<const T *>(h.data) + p.token * h.token_stride + p.head * h.head_stride + col, c.d - col, x);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (col + i < c.d) {
                bad |= !(fabsf(x[i]) <= 3.402823466e38f);
                mn = fminf(mn, x[i]);
                mx = fmaxf(mx, x[i]);
            }
    }
#pragma unroll
    for (int m = 1; m < LPR; m *= 2) {
        mn = fminf(mn, __shfl_xor(mn, m));
        mx = fmaxf(mx, __shfl_xor(mx, m));
        bad |= __shfl_xor(bad, m);
    }
    if (!p.there) return;
    constexpr float kTop = (1 << BITS) - 1;
    const float span = mx - mn;
    float inv = kTop / span, scale = span / kTop;
    if (!(fabsf(inv) <= 3.402823466e38f)) inv = scale = 0.f;
    if (bad || !(span <= 3.402823466e38f)) {
        mn = scale = NAN;
        inv = 0.f;
    }
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float f = fminf(fmaxf(rintf((x[i] - mn) * inv), 0.f), kTop);  // (a NaN becomes 0)
        q[i] = col + i < c.d ? (uint32_t)f : 0u;
    }
    uint8_t *codes = p.block + c.codes(p.which) + p.slot * c.rb;
    constexpr int kBytes = BITS;  // of 8 codes
    if (sub * kBytes < c.rb) {
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
        float *f = reinterpret_cast<float *>(p.block + c.floats(p.which)) + p.slot;
        f[0] = scale;
        f[c.ps()] = mn;
    }
}

template <typename T, int BITS, int LPR>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CachePages c, CacheBatch b, T *k, T *v) {
    int64_t row;
    bool in_call;
    const RowPlace p = place_row<LPR>(c, b, row, in_call);
    const int sub = threadIdx.x % LPR, col = 8 * sub;
    if (!in_call || col >= c.d) return;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (p.there) {
        const uint8_t *codes = p.block + c.codes(p.which) + p.slot * c.rb;
        const float *f = reinterpret_cast<const float *>(p.block + c.floats(p.which)) + p.slot;
        const float scale = f[0], mn = f[c.ps()];
        if constexpr (BITS == 8) {
            const uint2 w = *reinterpret_cast<const uint2 *>(codes + 8 * sub);
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = fmaf((float)((i < 4 ? w.x : w.y) >> 8 * (i & 3) & 255), scale, mn);
        } else {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + 4 * sub);
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = fmaf((float)(w >> 4 * i & 15), scale, mn);
        }
    }
    store8_any((p.which ? v : k) + (p.token * c.heads + p.head) * c.d + col, c.d - col, x);
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

// workgroups of `b.tokens` tokens; below 2^31, as the entry points see to
unsigned row_blocks(const CachePages &c, const CacheBatch &b, int lpr) {
    const int64_t rows = b.tokens * 2 * c.heads, per = kThreads / lpr;
    return (unsigned)((rows + per - 1) / per);
}

}  // namespace

#define BF_BY_TYPE(CALL)                              \
    if (dtype == BIFEAT_F32) { CALL(float); }         \
    else if (dtype == BIFEAT_F16) { CALL(Half16); }   \
    else { CALL(Brain16); }

hipError_t launch_cache_write(const CachePages &c, const CacheBatch &b, const HeadRows &k, const HeadRows &v, int bits, int dtype,
                              hipStream_t s) {
    const int lpr = lanes_per_row(c.d);
    const unsigned grid = row_blocks(c, b, lpr);
#define BF_GO(T, LPR)                                                                     \
    if (bits == 8) cache_write_kernel<T, 8, LPR><<<grid, kThreads, 0, s>>>(c, b, k, v);   \
    else cache_write_kernel<T, 4, LPR><<<grid, kThreads, 0, s>>>(c, b, k, v)
#define BF_LPR(T) if (lpr == 8) { BF_GO(T, 8); } else if (lpr == 16) { BF_GO(T, 16); } else { BF_GO(T, 32); }
    BF_BY_TYPE(BF_LPR)
#undef BF_GO
    return hipGetLastError();
}

hipError_t launch_cache_read(const CachePages &c, const CacheBatch &b, void *k, void *v, int bits, int dtype, hipStream_t s) {
    const int lpr = lanes_per_row(c.d);
    const unsigned grid = row_blocks(c, b, lpr);
#define BF_GO(T, LPR)                                                                                       \
    if (bits == 8) cache_read_kernel<T, 8, LPR><<<grid, kThreads, 0, s>>>(c, b, (T *)k, (T *)v);            \
    else cache_read_kernel<T, 4, LPR><<<grid, kThreads, 0, s>>>(c, b, (T *)k, (T *)v)
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
