// Attention of new tokens over the paged cache.
#include "cache.hpp"

namespace bf {
namespace {

// A wave a query row: 64 positions a step, one a lane; then a lane 4 of the values' columns.
template <typename T, int BITS>
__global__ __launch_bounds__(64) void cache_attend_kernel(AttendCall a) {
    __shared__ float qs[256];
    const CachePages &c = a.c;
    const int Hq = c.heads * a.group, lane = threadIdx.x;
    const int64_t t = blockIdx.x / Hq;
    const int hq = (int)(blockIdx.x % Hq), head = hq / a.group;
    const int seq = sequence_of(a.b, t);
    const int64_t len = a.b.length(seq, c.ps_log2), pos = len - a.b.count(seq) + (t - a.b.first(seq));
    const T *q = static_cast<const T *>(a.q.data) + t * a.q.token_stride + hq * a.q.head_stride;
    float qsum = 0.f;
    for (int j = lane; j < c.d; j += 64) {
        qs[j] = to_float(q[j]);
        qsum += qs[j];
    }
    for (int m = 1; m < 64; m *= 2) qsum += __shfl_xor(qsum, m);
    __syncthreads();
    float top = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    const int64_t prefix = a.prefix ? a.prefix[seq] : 0;
    int64_t end = pos + 1 > prefix ? pos + 1 : prefix;
    if (end > len) end = len;
    if (pos < 0) end = 0;
    const float slope = a.slopes ? a.slopes[hq] : 0.f;
    for (int64_t j0 = 0; j0 < end; j0 += 64) {
        const int64_t j = j0 + lane;
        const bool seen = j < end && ((j <= pos && (a.window == 0 || j > pos - a.window)) || j < prefix);
        float x = -INFINITY;
        if (seen) {
            const uint8_t *block = c.block(a.b.tables[seq * a.b.width + (j >> c.ps_log2)], head);
            const int slot = (int)(j & (c.ps() - 1));
            const uint8_t *codes = block + c.codes(0) + (int64_t)slot * c.rb;
            const float *f = reinterpret_cast<const float *>(block + c.floats(0)) + slot;
            float dot = 0.f;
            for (int i = 0; i < c.d; i++) dot += qs[i] * (float)(codes[i * BITS / 8] >> (i * BITS % 8) & ((1 << BITS) - 1));
            x = a.scale * (f[0] * dot + f[c.ps()] * qsum);
            if (a.softcap > 0.f) x = a.softcap * tanhf(x / a.softcap);
            x += slope * (float)(j - pos);
        }
        float m = x;
        for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
        if (!__any(seen)) continue;
        const float now = fmaxf(fmaxf(top, m), -1e30f), keep = expf(top - now), p = seen ? expf(x - now) : 0.f;
        top = now;
        float s = p;
        for (int o = 1; o < 64; o *= 2) s += __shfl_xor(s, o);
        sum = sum * keep + s;
        for (int k = 0; k < 4; k++) acc[k] *= keep;
        for (int i = 0; i < 64; i++) {
            const float w = __shfl(p, i);
            if (!__shfl((int)seen, i)) continue;
            const int64_t ji = j0 + i;
            const uint8_t *block = c.block(a.b.tables[seq * a.b.width + (ji >> c.ps_log2)], head);
            const int slot = (int)(ji & (c.ps() - 1));
            const uint8_t *codes = block + c.codes(1) + (int64_t)slot * c.rb;
            const float *f = reinterpret_cast<const float *>(block + c.floats(1)) + slot;
            for (int k = 0; k < 4; k++) {
                const int col = lane + 64 * k;
                if (col < c.d) acc[k] += w * fmaf((float)(codes[col * BITS / 8] >> (col * BITS % 8) & ((1 << BITS) - 1)), f[0], f[c.ps()]);
            }
        }
    }
    T *out = static_cast<T *>(a.out) + (t * Hq + hq) * c.d;
    for (int k = 0; k < 4; k++) {
        const int col = lane + 64 * k;
        if (col < c.d) out[col] = from_float<T>(sum != 0.f ? acc[k] / sum : 0.f);
    }
}

}  // namespace

hipError_t launch_cache_attend(bifeat_cache *h, const AttendCall &a) {
    const unsigned grid = (unsigned)(a.b.tokens * a.c.heads * a.group);
#define BF_GO(T)                                                                    \
    if (h->spec.bits == 8) cache_attend_kernel<T, 8><<<grid, 64, 0, a.s>>>(a);      \
    else cache_attend_kernel<T, 4><<<grid, 64, 0, a.s>>>(a)
    if (a.dtype == BIFEAT_F32) { BF_GO(float); }
    else if (a.dtype == BIFEAT_F16) { BF_GO(Half16); }
    else { BF_GO(Brain16); }
#undef BF_GO
    return hipGetLastError();
}

bool ensure_partial(bifeat_cache *, hipStream_t) { return true; }

}  // namespace bf
