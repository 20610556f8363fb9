// New tokens' keys turned to their positions on their way into the paged cache, and their queries beside them.
#include <algorithm>

#include "cache_rows.hpp"

namespace bf {
namespace {

// Column pair i of a row is turned by the angle a = p f_i, p the token's position: (u, w) becomes (u cos a - w sin a, u sin a + w cos a),
// times a scale.  Angle, cosine, sine and the turned columns are 64-bit numbers: p f_i is exact below 2^29 positions, and a key's column comes
// to its quantiser as the 32-bit number next to the exact one, so that codes are the definition's (an error of 2^-53 moves a rounding to 32
// bits once in 2^29 columns, where one of 2^-24 moves a level in 10 000).
struct Turn {
    const float *frequencies;
    int pairs;
    bool interleaved;  // pairs are columns 2 i and 2 i + 1, else i and i + pairs
    double scale;
};

// The eight columns from `col` of a row, turned.
template <typename T>
__device__ inline void turn8(const Turn &t, const T *row, int col, int d, const double *cs, float (&x)[8]) {
    if (col >= 2 * t.pairs) return;
    const double *cosine = cs, *sine = cs + t.pairs;
    if (t.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const int pair = (col + i) / 2;
            if (pair < t.pairs) {
                const double u = x[i], w = x[i + 1], c = cosine[pair], s = sine[pair];
                x[i] = (float)(u * c - w * s);
                x[i + 1] = (float)(u * s + w * c);
            }
        }
        return;
    }
    float other[8];  // the columns' partners
    if (t.pairs % 8 == 0) {
        const int at = col < t.pairs ? col + t.pairs : col - t.pairs;
        load8_any(row + at, d - at, other);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int c = col + i;
            other[i] = c < 2 * t.pairs ? to_float(row[c < t.pairs ? c + t.pairs : c - t.pairs]) : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int c = col + i;
        if (c < t.pairs) x[i] = (float)((double)x[i] * cosine[c] - (double)other[i] * sine[c]);
        else if (c < 2 * t.pairs) x[i] = (float)((double)other[i] * sine[c - t.pairs] + (double)x[i] * cosine[c - t.pairs]);
    }
}

template <typename T, int BITS, int LPR>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CachePages c, CacheBatch b, HeadRows q, int query_heads, HeadRows k, HeadRows v,
                                                                Turn turn, T *out, int per) {
    __shared__ Places places;
    extern __shared__ double turns[];  // [token][cosines, sines]
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const int count = b.tokens - t0 < per ? (int)(b.tokens - t0) : per;
    find_places(c, b, t0, count, places);
    for (int i = threadIdx.x; i < count * turn.pairs; i += kThreads) {
        const int token = i / turn.pairs, pair = i - token * turn.pairs;
        double s, co;
        sincos((double)places.position[token] * (double)turn.frequencies[pair], &s, &co);
        turns[2 * token * turn.pairs + pair] = co * turn.scale;
        turns[(2 * token + 1) * turn.pairs + pair] = s * turn.scale;
    }
    __syncthreads();
    const int sub = threadIdx.x % LPR, col = 8 * sub, per_token = query_heads + 2 * c.heads, rows = count * per_token;
    for (int r0 = threadIdx.x / 64 * (64 / LPR); r0 < rows; r0 += kThreads / LPR) {
        const int r = r0 + threadIdx.x % 64 / LPR, token = r % count, which_head = r / count;
        const bool inside = r < rows, query = which_head < query_heads, value = which_head >= query_heads + c.heads;
        const int head = query ? which_head : value ? which_head - query_heads - c.heads : which_head - query_heads;
        const bool real = inside && places.page[token] >= 0;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = 0.f;
        if (real && col < c.d) {
            const HeadRows &h = query ? q : value ? v : k;
            const T *row = static_cast<const T *>(h.data) + (t0 + token) * h.token_stride + head * h.head_stride;
            load8_any(row + col, c.d - col, x);
            if (!value) turn8(turn, row, col, c.d, turns + 2 * token * turn.pairs, x);
        }
        if (inside && query && col < c.d) store_any<8, false>(out + ((t0 + token) * query_heads + head) * c.d + col, c.d - col, x);
        const int cached = query ? 0 : head;
        write_row<BITS, LPR>(c, x, real && !query, c.pages + (real ? places.page[token] : 0) + cached * c.head_bytes, value, places.slot[token]);
    }
}

}  // namespace

hipError_t launch_cache_append(const CachePages &c, const CacheBatch &b, const AppendCall &a) {
    const int lpr = lanes_per_row(c.d);
    const int per = (int)std::max<int64_t>(1, std::min<int64_t>(kTokens, b.tokens / 2048));
    const unsigned grid = (unsigned)((b.tokens + per - 1) / per);
    const Turn turn{a.frequencies, a.pairs, a.interleaved, a.scale};
    const size_t room = (size_t)per * a.pairs * 2 * sizeof(double);
#define BF_GO(T, BITS, LPR)                                                                                                         \
    cache_append_kernel<T, BITS, LPR><<<grid, kThreads, room, a.s>>>(c, b, a.q, a.query_heads, a.k, a.v, turn, (T *)a.out, per)
#define BF_LPR(T, BITS)                     \
    if (lpr == 8) { BF_GO(T, BITS, 8); }    \
    else if (lpr == 16) { BF_GO(T, BITS, 16); } \
    else { BF_GO(T, BITS, 32); }
#define BF_BITS(T) if (a.bits == 8) { BF_LPR(T, 8) } else { BF_LPR(T, 4) }
    if (a.dtype == BIFEAT_F32) { BF_BITS(float) }
    else if (a.dtype == BIFEAT_F16) { BF_BITS(Half16) }
    else { BF_BITS(Brain16) }
#undef BF_GO
#undef BF_LPR
#undef BF_BITS
    return hipGetLastError();
}

}  // namespace bf
