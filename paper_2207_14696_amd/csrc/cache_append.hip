// New tokens' keys turned to their positions on their way into the paged cache, and their queries beside them.
#include <algorithm>

#include "cache_rows.hpp"

namespace bf {
namespace {

// Column pair i of a row is turned by the angle a = p f_i, p the token's position: (u, w) becomes (u cos a - w sin a, u sin a + w cos a),
// times a scale.  Angle, cosine, sine and the turned columns are 64-bit numbers: p f_i is exact below 2^29 positions (and the number next to it up to the last), and a
// key's column comes to its quantiser as the 32-bit number next to the exact one, so that codes are the definition's (an error of 2^-53 moves a rounding to 32
// bits once in 2^29 columns, where one of 2^-24 moves a level in 10 000).
struct Turn {
    const float *frequencies;
    int pairs;
    bool interleaved;  // pairs are columns 2 i and 2 i + 1, else i and i + pairs
    double scale;
};

// Sine and cosine of an angle below 2^50 in size, off by less than 2^-51, of others NaN: what is left of it after the nearest multiple of a quarter turn (whose
// product with a quarter turn of 106 bits the fused multiply-adds take off with one rounding each), by the series at zero as far as r^17 and r^16
// (the next terms are below 2^-58 of 1).
__device__ inline void sine_and_cosine(double angle, double &sine, double &cosine) {
    const bool far = !(fabs(angle) < 0x1p50);
    const double n = far ? 0.0 : rint(angle * 0x1.45f306dc9c883p-1);                                       // 2 / pi
    const double r = fma(-n, 0x1.1a62633145c07p-54, fma(-n, 0x1.921fb54442d18p+0, angle)), z = r * r;     // pi / 2 in two pieces
    double s = 1.0 / 355687428096000.0, c = 1.0 / 20922789888000.0;
    s = fma(z, s, -1.0 / 1307674368000.0);
    c = fma(z, c, -1.0 / 87178291200.0);
    s = fma(z, s, 1.0 / 6227020800.0);
    c = fma(z, c, 1.0 / 479001600.0);
    s = fma(z, s, -1.0 / 39916800.0);
    c = fma(z, c, -1.0 / 3628800.0);
    s = fma(z, s, 1.0 / 362880.0);
    c = fma(z, c, 1.0 / 40320.0);
    s = fma(z, s, -1.0 / 5040.0);
    c = fma(z, c, -1.0 / 720.0);
    s = fma(z, s, 1.0 / 120.0);
    c = fma(z, c, 1.0 / 24.0);
    s = fma(z, s, -1.0 / 6.0);
    c = fma(z, c, -0.5);
    s = fma(r * z, s, r);
    c = fma(z, c, 1.0);
    const long long quarter = (long long)n;
    const double a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
    sine = far ? NAN : quarter & 2 ? -a : a;
    cosine = far ? NAN : (quarter + 1) & 2 ? -b : b;
}

// What the widths of rows and turns allow: any; whole eights of columns, pairs next to each other (or none); whole eights that are paired with whole eights.
enum Widths { kAny, kNeighbours, kHalves };

// Eight columns of a row from `col`, and those that they are paired with where these are not next to them.
template <typename T, Widths W>
struct Fetched {
    Columns<T> x, other;
};
template <typename T>
struct Fetched<T, kNeighbours> {
    Columns<T> x;
};
// A lane without columns is given the address of some that are there: loads that no branch leads to are all asked for before any is waited for.
template <typename T, Widths W>
__device__ inline Fetched<T, W> fetch(const Turn &t, const T *row, int col, int d, bool turned) {
    Fetched<T, W> f;
    if constexpr (W != kAny) {
        f.x = load_columns(row + (col < d ? col : 0));
        if constexpr (W == kHalves) f.other = load_columns(row + (turned && col < 2 * t.pairs ? (col < t.pairs ? col + t.pairs : col - t.pairs) : col < d ? col : 0));
    } else {
        T v[8] = {}, w[8] = {};
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (col + i < d) v[i] = row[col + i];
            if (turned && !t.interleaved && col + i < 2 * t.pairs) w[i] = row[col + i < t.pairs ? col + i + t.pairs : col + i - t.pairs];
        }
        __builtin_memcpy(f.x.w, v, sizeof(f.x));
        __builtin_memcpy(f.other.w, w, sizeof(f.other));
    }
    return f;
}
template <typename T>
__device__ inline void to_floats(const Columns<T> &c, float (&x)[8]) {
    T v[8];
    __builtin_memcpy(v, c.w, sizeof(c));
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = to_float(v[i]);
}

// They turned, in numbers of type F; cs: the token's cosines, then its sines.
template <typename F, typename T, Widths W>
__device__ inline void turn8(const Turn &t, const Fetched<T, W> &f, int col, const F *cs, float (&x)[8]) {
    if (col >= 2 * t.pairs) return;
    const F *cosine = cs, *sine = cs + t.pairs;
    if (W == kNeighbours || (W == kAny && t.interleaved)) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const int pair = (col + i) / 2;
            if (pair < t.pairs) {
                const F u = x[i], w = x[i + 1], c = cosine[pair], s = sine[pair];
                x[i] = (float)(u * c - w * s);
                x[i + 1] = (float)(u * s + w * c);
            }
        }
        return;
    }
    if constexpr (W != kNeighbours) {
        float other[8];
        to_floats(f.other, other);
        if constexpr (W == kHalves) {
            const bool first = col < t.pairs;
            const int pair = first ? col : col - t.pairs;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const F s = (F)(first ? -other[i] : other[i]) * sine[pair + i];
                x[i] = (float)((F)x[i] * cosine[pair + i] + s);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int c = col + i, pair = c < t.pairs ? c : c - t.pairs;
                if (c < 2 * t.pairs) {
                    const F s = (F)(c < t.pairs ? -other[i] : other[i]) * sine[pair];
                    x[i] = (float)((F)x[i] * cosine[pair] + s);
                }
            }
        }
    }
}

// A workgroup takes up to kTokens tokens: a wave the rows of keys and values that 64 lanes take, a token's after another's as in their page, then those of
// queries, a head's after another's as in the projection; the next rows are on their way while these are turned and quantised, the first of them
// while the tokens' places and turns are made.
// Queries of 16 bits are turned in 32, by cosines and sines rounded to 32: 2^-23 of the pair, beside their own 2^-11 or 2^-8.
template <typename T, int BITS, int LPR, Widths W>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CachePages c, CacheBatch b, HeadRows q, int query_heads, HeadRows k, HeadRows v,
                                                                Turn turn, T *out, int per, uint32_t per_inverse) {
    typedef std::conditional_t<sizeof(T) == 4, double, float> Wide;  // of queries
    __shared__ Places places;
    extern __shared__ double turns[];  // [token][cosines, sines], and then the same rounded
    constexpr int kRowsAtOnce = 64 / LPR, kWaves = kThreads / 64;
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const int count = b.tokens - t0 < per ? (int)(b.tokens - t0) : per;
    const int sub = threadIdx.x % LPR, col = 8 * sub, mine = threadIdx.x % 64 / LPR, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int rows = per * 2 * c.heads, items = (rows + kRowsAtOnce - 1) / kRowsAtOnce;
    struct Row {
        int token, head;
        bool value, real;
    };
    const auto row_of = [&](int item) {
        const int i = item * kRowsAtOnce + mine, h = per == 1 ? i : (int)__umulhi(i, per_inverse), token = i - h * per;  // i / per
        return i < rows && token < count ? Row{token, h < c.heads ? h : h - c.heads, h >= c.heads, true} : Row{0, 0, false, false};
    };
    const auto get = [&](const Row &r) {  // (of none: the first key)
        const HeadRows h{r.value ? v.data : k.data, r.value ? v.token_stride : k.token_stride, r.value ? v.head_stride : k.head_stride};
        return fetch<T, W>(turn, static_cast<const T *>(h.data) + (t0 + r.token) * h.token_stride + r.head * h.head_stride, col, c.d, !r.value);
    };
    int item = wave;
    Row row = row_of(item);
    Fetched<T, W> now = get(row);
    find_places(c, b, t0, count, places);
    Wide *wide = reinterpret_cast<Wide *>(turns + (sizeof(T) == 4 ? 0 : 2 * per * turn.pairs));
    for (int i = threadIdx.x; i < count * turn.pairs; i += kThreads) {
        const int token = i / turn.pairs, pair = i - token * turn.pairs, at = 2 * token * turn.pairs + pair;
        double s, co;
        sine_and_cosine((double)places.position[token] * (double)turn.frequencies[pair], s, co);
        turns[at] = co * turn.scale;
        turns[at + turn.pairs] = s * turn.scale;
        if constexpr (sizeof(T) == 2) {
            wide[at] = (float)(co * turn.scale);
            wide[at + turn.pairs] = (float)(s * turn.scale);
        }
    }
    __syncthreads();
    for (; item < items; item += kWaves) {
        const Row next = row_of(item + kWaves);
        const Fetched<T, W> coming = get(next);
        const bool real = row.real && places.page[row.token] >= 0;
        float x[8];
        to_floats(now.x, x);
        if (!row.value) turn8(turn, now, col, turns + 2 * row.token * turn.pairs, x);
        write_row<BITS, LPR>(c, x, real, c.pages + places.page[row.token] + row.head * c.head_bytes, row.value, places.slot[row.token]);
        row = next;
        now = coming;
    }
    if (query_heads == 0) return;
    // the queries: `at` counts a token's rows, by as many as the waves take at once
    const int head0 = wave * kRowsAtOnce + mine;
    const int64_t step = (int64_t)kWaves * kRowsAtOnce;
    for (int token = 0; token < count; token++) {
        const T *from = static_cast<const T *>(q.data) + (t0 + token) * q.token_stride + head0 * q.head_stride;
        T *to = out + ((t0 + token) * query_heads + head0) * c.d + col;
        const bool real = places.page[token] >= 0;
        const Wide *cs = wide + 2 * token * turn.pairs;
        for (int head = head0; head < query_heads; head += step) {
            const Fetched<T, W> f = fetch<T, W>(turn, from, col, c.d, true);
            float x[8];
            to_floats(f.x, x);
            turn8(turn, f, col, cs, x);
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = real ? x[e] : 0.f;
            if (col < c.d) store_any<8, false>(to, W == kAny ? c.d - col : 8, x);
            from += step * q.head_stride;
            to += step * c.d;
        }
    }
}

}  // namespace

hipError_t launch_cache_append(const CachePages &c, const CacheBatch &b, const AppendCall &a) {
    const int lpr = lanes_per_row(c.d);
    const int per = (int)std::max<int64_t>(1, std::min<int64_t>(kTokens, b.tokens / 2048));
    const unsigned grid = (unsigned)((b.tokens + per - 1) / per);
    const Turn turn{a.frequencies, a.pairs, a.interleaved, a.scale};
    const size_t room = (size_t)per * a.pairs * 2 * (sizeof(double) + (a.dtype == BIFEAT_F32 ? 0 : sizeof(float)));
    const uint32_t per_inverse = (uint32_t)(((1ull << 32) + per - 1) / per);  // (of 1: unused)
    const Widths widths = c.d % 8 || (!a.interleaved && a.pairs % 8) ? kAny : a.interleaved || !a.pairs ? kNeighbours : kHalves;
#define BF_RUN(T, BITS, LPR, W)                                                                                                         \
    cache_append_kernel<T, BITS, LPR, W><<<grid, kThreads, room, a.s>>>(c, b, a.q, a.query_heads, a.k, a.v, turn, (T *)a.out, per, per_inverse)
#define BF_GO(T, BITS, LPR)                                   \
    if (widths == kAny) BF_RUN(T, BITS, LPR, kAny);           \
    else if (widths == kHalves) BF_RUN(T, BITS, LPR, kHalves); \
    else BF_RUN(T, BITS, LPR, kNeighbours)
#define BF_LPR(T, BITS)                     \
    if (lpr == 8) { BF_GO(T, BITS, 8); }    \
    else if (lpr == 16) { BF_GO(T, BITS, 16); } \
    else { BF_GO(T, BITS, 32); }
#define BF_BITS(T) if (a.bits == 8) { BF_LPR(T, 8) } else { BF_LPR(T, 4) }
    if (a.dtype == BIFEAT_F32) { BF_BITS(float) }
    else if (a.dtype == BIFEAT_F16) { BF_BITS(Half16) }
    else { BF_BITS(Brain16) }
#undef BF_RUN
#undef BF_GO
#undef BF_LPR
#undef BF_BITS
    return hipGetLastError();
}

}  // namespace bf
