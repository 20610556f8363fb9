// Attention over the paged cache: how the work is dealt to workgroups, and what the kernels share.
//
// Mathematics.  A cached row is x = mn + code * s.  Products with the keys and sums of the values are taken on the codes:
//     q . k_t = s_t (q . code_t) + mn_t sum(q)            sum_t p_t v_t = sum_t (p_t s_t) code_t + sum_t p_t mn_t
// so that the matrix cores see whole numbers, which fp16 holds exactly, and nothing is decoded.  A code's bits are read as
// an fp16 number as they stand: a subnormal, code * 2^-24, which the matrix cores of gfx950 multiply as it is (the factor is
// taken out in 32 bits).  One byte permutation makes two operands of two 8-bit codes; of 4-bit values' codes a mask makes two, or
// two times 16, which is taken out of the sum; those of keys are all times 16 (see key_of4).
// The values' codes are weighted about the middle of their range (c = mn + 2^(bits-1) s): what a weight's rounding to fp16
// is off by then meets at most half a row's range.
#pragma once

#include "cache.hpp"

namespace bf {

constexpr int kRowsR = 16, kRowsTok = 128;    // items and units of the kernel for few rows
// Tiles of 16 rows a wave in the kernel for many.  None of these kernels may spill vector registers: this compiler (clang 22
// for gfx950) has been seen to place such a spill at the join of a divergent branch before it restores the lanes' mask, so
// that the lanes outside the branch got their values back wrong.  Two tiles where sums and queries leave room for it.
constexpr int chunk_tiles(int dp, int np) { return dp == 64 || (dp == 128 && np == 1) ? 2 : 1; }
constexpr float kLog2e = 1.4426950408889634f;
// A row's weights are p = 2^(x - top), and fp16 gets p * s: `top`, a whole number, follows the largest x + log2(size), with the
// scale s of the position's values for its size.  It may lag (p * size up to 2^15) and is brought up for all lanes of a row together, to
// leave them 2^8.  A scale below 2^-80 (0 where the values are one) would let p grow without bound, and p * mn with it: such a position's
// size is 2^-80, or its values' by 2^24 where that is more, so that p stays within 2^95 and p * mn within 2^39, which leaves 2^30 positions
// room.  Steps that have one are sent down the seldom taken branch that brings `top` up; nothing else is asked of the others.  From 2^-80 on
// scales need no such care: written values of which two differ have s > mn 2^-32.
constexpr float kLeastScale = 8.271806125530277e-25f;  // 2^-80
// (of the middle code's value, which is within 2^7 s of mn)
__device__ inline float size_of(float s, float middle) { return s < kLeastScale ? fmaxf(fabsf(middle) * 5.9604644775390625e-8f, kLeastScale) : s; }
// What happens to scores, a kernel's MODE: nothing, a bias by distance, a cap (and a bias): the first form of cap_all alone, or both
enum { kPlain = 0, kBiased = 1, kCappedFirst = 2, kCapped = 3 };
inline int mode_of(const AttendCall &a) {
    if (a.softcap > 0.f) return a.dtype != BIFEAT_F32 && a.softcap <= 64.f ? kCappedFirst : kCapped;
    return a.slopes ? kBiased : kPlain;
}
constexpr float kNothing = -1e30f;  // running maximum where nothing was seen: below any score, and finite

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

// Work: an item is R query rows of a sequence and a cached head (row r: new token r / group, query head r % group of the
// head's), a unit is TOK positions of the cache that an item looks at.  The units of all items, in the order of heads,
// then sequences, then rows, are dealt evenly to `nw` workgroups, each a run of them; contexts of any mixture of
// lengths so keep all of them busy.  An item that several workgroups share is joined by a second kernel.
struct PartOf {  // where a workgroup begins
    int head, seq, rt;
    int unit, units;  // the first unit it has of the item, and the item's
    int nw;           // workgroups that have units (0: this one has none)
    int start, all;   // units before it, and of the call
    int rows;         // of the item
    int64_t token;    // the sequence's first of the call
};
struct AttendPlan {
    int items;       // per head; of a ragged batch with numbers left free (see first_item)
    int nw;
    int least;       // units that a workgroup has at least (see workgroups_of)
    // null: a workgroup has one item, all of it (contexts are short, or there is no workspace)
    float *partial;  // [nw][2]: of an item begun before / not ended by a workgroup sums [R][DP], reference [R], sum of weights [R]
    PartOf *begins;  // [nw]
};

// Workgroups of a call with `all` units: as many as run at a time (most), fewer where each would have less than `least` units;
// least 4: 2 will do where units are fewer than 512.  What workgroups leave to be joined costs more than a few units one after another:
// 16 rows of each of 8 sequences of 1024 on 8 heads of 128 (512 units) took 30 us by a unit each, 22 by two; 64 rows (1024 units,
// kernel for many) 47 by two, 39 by four; 64 rows of one of 512 (64 units) 26.5 by one, 26.7 by two, 31 by four.
__host__ __device__ inline int workgroups_of(int64_t all, int least, int most) {
    const int64_t n = least < 4 ? all / least : all < 512 ? all / 2 : all < 1024 ? 256 : all / 4;
    return n > most ? most : n > 1 ? (int)n : all > 0;
}

// `all` units over nw workgroups, nw <= all: the first all % nw have one more than the others
__device__ inline int start_of(int w, int all, int nw) { return w * (all / nw) + (w < all % nw ? w : all % nw); }
__device__ inline int workgroup_of(int unit, int all, int nw) {
    const int q = all / nw, r = all % nw;
    return unit < r * (q + 1) ? unit / (q + 1) : r + (unit - r * (q + 1)) / q;
}

// Sequence b's items have numbers from first_item(b) on.  In a ragged batch floor(rows before it / R) + b leaves every
// sequence room for its own, rounded up, without a sum over the batch.
template <int R>
__device__ inline int first_item(const AttendCall &a, int b) {
    if (!a.b.indptr) return b * ((a.b.n * a.group + R - 1) / R);
    return (int)(a.b.indptr[b] * a.group / R) + b;
}

// What an item's rows see.
struct View {
    int len, n;          // the sequence's
    int first, last;     // positions of the item's first and last query
    int prefix;
    int skip_at, skip;   // units: from the skip_at-th on, `skip` are left out
    int units;
};

template <int R, int TOK>
__device__ inline View view_of(const AttendCall &a, int b, int rt) {
    View v;
    v.len = (int)a.b.length(b, a.c.ps_log2);
    v.n = (int)a.b.count(b);
    const int rows = v.n * a.group;
    if (rt * R >= rows) {
        v.first = v.last = v.prefix = v.skip_at = v.skip = v.units = 0;
        return v;
    }
    const int end_row = rt * R + R < rows ? rt * R + R : rows;
    v.first = v.len - v.n + rt * R / a.group;
    v.last = v.len - v.n + (end_row - 1) / a.group;
    int64_t pre = a.prefix ? a.prefix[b] : 0;
    v.prefix = pre < 0 ? 0 : pre > v.len ? v.len : (int)pre;
    int end = v.last + 1 > v.prefix ? v.last + 1 : v.prefix;
    if (v.last < 0) end = 0;
    const int low = a.window ? v.first - a.window + 1 : 0;
    const int total = (end + TOK - 1) / TOK, from = low > 0 ? low / TOK : 0;
    v.skip_at = (v.prefix + TOK - 1) / TOK;
    v.skip = from < total ? from - v.skip_at : total - v.skip_at;
    if (v.skip < 0) v.skip = 0;
    v.units = total - v.skip > 1 ? total - v.skip : 1;  // an item that sees nothing still has its zeros to write
    return v;
}

// The same value in all lanes, in a scalar register.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    return (int64_t)(uint32_t)uniform((int)x) | (int64_t)uniform((int)(x >> 32)) << 32;
}
__device__ inline View uniform(const View &v) {
    return {uniform(v.len), uniform(v.n), uniform(v.first), uniform(v.last), uniform(v.prefix), uniform(v.skip_at), uniform(v.skip), uniform(v.units)};
}

struct Place {
    int seq, rt;  // an item: its sequence, its number in it
    int unit;     // of the item
};

// The sequence that item `i` of a head belongs to.
template <int R>
__device__ inline int sequence_of_item(const AttendCall &a, int i) {
    if (!a.b.indptr) return i / ((a.b.n * a.group + R - 1) / R);
    int lo = 0, hi = a.b.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first_item<R>(a, mid) <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Deals the units: workgroup w's are [*start, *end) of the call's, the first of them at *at.  All threads of a workgroup;
// sh: 16 ints.
template <int R, int TOK>
__device__ inline void locate(const AttendCall &a, const AttendPlan &p, int w, int *start, int *end, int *head, Place *at, int *sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    if (!p.partial) {
        w += (int)(gridDim.x * blockIdx.y);  // (see grid_of)
        *start = *end = 0;
        if (w >= p.items * a.c.heads) return;
        const int item = w % p.items;
        at->seq = uniform(sequence_of_item<R>(a, item));
        at->rt = uniform(item - first_item<R>(a, at->seq));
        at->unit = 0;
        *head = w / p.items;
        *end = uniform(view_of<R, TOK>(a, at->seq, at->rt).units);
        return;
    }
    // a thread sums the units of some of a head's items
    const int per = (p.items + (int)blockDim.x - 1) / (int)blockDim.x;
    const int i0 = tid * per, i1 = i0 + per < p.items ? i0 + per : p.items;
    int sum = 0;
    const int seq = i0 < i1 ? sequence_of_item<R>(a, i0) : 0;
    int s = seq, next = i0 < i1 ? first_item<R>(a, s + 1) : 0;
    for (int i = i0; i < i1; i++) {
        while (i >= next && s + 1 < a.b.B) next = first_item<R>(a, ++s + 1);
        sum += view_of<R, TOK>(a, s, i - first_item<R>(a, s)).units;
    }
    int upto = sum;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int x = __shfl_up(upto, m);
        if (lane >= m) upto += x;
    }
    if (lane == 63) sh[wave] = upto;
    __syncthreads();
    int total = 0, before = upto - sum;
    for (int k = 0; k < waves; k++) {
        if (k < wave) before += sh[k];
        total += sh[k];
    }
    total = __builtin_amdgcn_readfirstlane(total);
    const int all = total * a.c.heads, nw = workgroups_of(all, p.least, p.nw);  // (none has nothing between two that have)
    if (w >= nw) {
        *start = *end = 0;
        if (tid == 0) p.begins[w].nw = 0;
        return;
    }
    *start = start_of(w, all, nw);
    *end = start_of(w + 1, all, nw);
    *head = *start / total;
    const int want = *start - *head * total;
    if (want >= before && want < before + sum) {
        int left = want - before;
        s = seq, next = first_item<R>(a, s + 1);
        for (int i = i0; i < i1; i++) {
            while (i >= next && s + 1 < a.b.B) next = first_item<R>(a, ++s + 1);
            const int rt = i - first_item<R>(a, s), u = view_of<R, TOK>(a, s, rt).units;
            if (left < u) {
                sh[8] = s, sh[9] = rt, sh[10] = left;
                const int rows = (int)a.b.count(s) * a.group - rt * R;
                p.begins[w] = {*head, s, rt, left, u, nw, *start, all, rows < R ? rows : R, a.b.first(s)};
                break;
            }
            left -= u;
        }
    }
    __syncthreads();
    at->seq = __builtin_amdgcn_readfirstlane(sh[8]);
    at->rt = __builtin_amdgcn_readfirstlane(sh[9]);
    at->unit = __builtin_amdgcn_readfirstlane(sh[10]);
}

// The next item that has units, of this head or the next.
template <int R>
__device__ inline void next_item(const AttendCall &a, int *head, Place *at) {
    at->unit = 0;
    at->rt++;
    while (at->rt * R >= uniform((int)a.b.count(at->seq)) * a.group) {
        at->rt = 0;
        if (++at->seq == a.b.B) {
            at->seq = 0;
            ++*head;
        }
    }
}

// Power of two that brings `top` to [2^to, 2^(to+1)) (within 2^-80 .. 2^80; 1 for 0).
__device__ inline float power_to(float top, int to) {
    int e = (int)(__builtin_bit_cast(uint32_t, top) >> 23 & 255) - 127;
    e = top > 0.f ? (e < -80 ? -80 : e > 80 ? 80 : e) : to;
    return __builtin_bit_cast(float, (uint32_t)(127 + to - e) << 23);
}

// codes -> fp16 operands ----------------------------------------------------------------------------------------------

// the bytes lo and hi of a as two halves
__device__ inline uint32_t bytes_of(uint32_t a, int lo) { return __builtin_amdgcn_perm(0u, a, 0x0c000c00u | lo | (lo + 1) << 16); }
// byte i of a, byte i of b as two halves
__device__ inline uint32_t pair_of(uint32_t a, uint32_t b, int i) { return __builtin_amdgcn_perm(b, a, 0x0c000c00u | i | (4 + i) << 16); }

struct Words4 { uint32_t w[4]; };
__device__ inline half8 operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(half8, Words4{{a, b, c, d}});
}

// Eight 4-bit codes of a key, all times 16: (0, 4), (1, 5), (2, 6), (3, 7).  Of subnormal operands the matrix cores lose the bits that a normal
// number would have in place of their leading zeros; with every other pair as it stands, two instructions fewer, scores were off by 2^-21.4
// of the sum of |q| |k| (root mean square), so by 2^-24, as of 8-bit codes (contexts of 131 072 in 4 bits 112.5 us, 115 so).
__device__ inline half8 key_of4(uint32_t w) {
    auto at = [](uint32_t x) { return x & 0x00f000f0u; };
    return operand(at(w << 4), at(w), at(w >> 4), at(w >> 8));
}

// Codes as whole numbers less their middle (4-bit ones' times 16 where they come so), for 32-bit queries: 1024 + code is the code's bits beside
// 1024's, and 1024 + middle is taken off exactly.  Sums of products of codes that are all positive leave 2^-24 of the codes' common part.
__device__ inline half8 centred(half8 bits, half8 top) {
    Words4 w = __builtin_bit_cast(Words4, bits);
#pragma unroll
    for (int i = 0; i < 4; i++) w.w[i] |= 0x64006400u;
    return __builtin_bit_cast(half8, w) - top;
}
__device__ inline half8 all_of(float x) {
    const _Float16 m = (_Float16)x;
    return half8{m, m, m, m, m, m, m, m};
}
// the unit of a product with a value's code: codes are subnormals, or (NP = 2) whole numbers; and with a key's, 4-bit ones times 16
template <int NP> constexpr float kUnit = NP == 2 ? 1.f : 16777216.f;
template <int BITS, int NP> constexpr float kKeyUnit = kUnit<NP> / (BITS == 4 ? 16 : 1);

// Loads from a head's block of a page, whose address all lanes share: a descriptor in scalar registers, a 32-bit offset a lane
// and one for all, where 64-bit addresses would take two vector registers and three vector instructions a load.  (The
// hardware gives zeros past the block's end, without a fetch: past any, if the block is not wanted.)
__device__ inline __amdgpu_buffer_rsrc_t block_buffer(const CachePages &c, int page, int head, bool wanted = true) {
    return __builtin_amdgcn_make_buffer_rsrc(c.block(page, head), 0, wanted ? (int)c.head_bytes : 0, 0x00027000);
}
// STREAMED: not kept in the caches
template <int N, bool STREAMED>
__device__ inline void load_bytes(__amdgpu_buffer_rsrc_t r, uint32_t each, uint32_t all, uint32_t *w) {
    constexpr int kPolicy = STREAMED ? 2 : 0;
    if constexpr (N == 16) {
        const auto q = __builtin_amdgcn_raw_buffer_load_b128(r, each, all, kPolicy);
        w[0] = q[0], w[1] = q[1], w[2] = q[2], w[3] = q[3];
    } else if constexpr (N == 8) {
        const auto q = __builtin_amdgcn_raw_buffer_load_b64(r, each, all, kPolicy);
        w[0] = q[0], w[1] = q[1];
    } else if constexpr (N == 4) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, each, all, kPolicy);
    } else if constexpr (N == 2) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b16(r, each, all, kPolicy);
    } else {
        w[0] = __builtin_amdgcn_raw_buffer_load_b8(r, each, all, kPolicy);
    }
}
// x, which nothing that is made of it is to leave this place: mask bits tested ahead of a branch that seldom needs them cost 16 of
// 50 instructions, and addresses worked out once for all items the registers that sums need.
__device__ inline uint32_t here(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Queries to LDS, as they are: rows row0 .. row0 + N - 1 of a sequence and cached head, zeros from column a.c.d and row `rows`
// on; by `threads` threads of which this is number `me`, in pieces of P columns (which divides a.c.d).  row0 < rows.  E: uint16_t or
// float.
template <int N, int DP, int STRIDE, int P, typename E>
__device__ inline void stage_pieces(const AttendCall &a, int64_t token0, int head, int row0, int rows, E *to, int me, int threads) {
    const E *q = static_cast<const E *>(a.q.data) + token0 * a.q.token_stride + (int64_t)head * a.group * a.q.head_stride;
    struct __attribute__((packed, aligned(sizeof(E)))) Piece { E v[P]; };
    struct __attribute__((aligned(P * sizeof(E)))) Slot { E v[P]; };
    constexpr int kPer = DP / P, kBatch = 8;  // pieces a row, and in flight
#pragma unroll 1
    for (int i0 = me; i0 < N * kPer; i0 += kBatch * threads) {
        Slot x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; k++) {
            const int i = i0 + k * threads, r = row0 + i / kPer, col = i % kPer * P;
            const bool there = i < N * kPer && r < rows && col < a.c.d;
            const int rr = there ? r : row0;
            const Piece y = *reinterpret_cast<const Piece *>(q + rr / a.group * a.q.token_stride + rr % a.group * a.q.head_stride + (there ? col : 0));
#pragma unroll
            for (int e = 0; e < P; e++) x[k].v[e] = there ? y.v[e] : (E)0;
        }
#pragma unroll
        for (int k = 0; k < kBatch; k++) {
            const int i = i0 + k * threads;
            if (i < N * kPer) *reinterpret_cast<Slot *>(to + i / kPer * STRIDE + i % kPer * P) = x[k];
        }
    }
}
template <int N, int DP, int STRIDE, typename E>
__device__ inline void stage_queries(const AttendCall &a, int64_t token0, int head, int row0, int rows, E *to, int me, int threads) {
    me = (int)here((uint32_t)me);
    if (a.c.d % 4 == 0) stage_pieces<N, DP, STRIDE, 4>(a, token0, head, row0, rows, to, me, threads);
    else stage_pieces<N, DP, STRIDE, 1>(a, token0, head, row0, rows, to, me, threads);
}
// 8 of them, and as floats
template <typename E>
struct __attribute__((aligned(8 * sizeof(E)))) Queries8 { E v[8]; };
template <typename E>
__device__ inline void floats_of(const Queries8<E> &q, bool half, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if constexpr (sizeof(E) == 4) x[i] = q.v[i];
        else x[i] = half ? to_float(Half16{q.v[i]}) : to_float(Brain16{q.v[i]});
    }
}
// (only of queries that see something: the others may hold anything)
__device__ inline float largest_finite(float most, const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) most = fmaxf(most, fabsf(x[i]) <= 3.402823466e38f ? fabsf(x[i]) : 0.f);
    return most;
}
// 8 columns as an operand beside 8 codes, which of 4 bits come as 0, 4, 1, 5, 2, 6, 3, 7.  Returns what they add up to.
template <int BITS, int NP>
__device__ inline float query_operand(const float (&x)[8], float up, half8 &hi8, half8 &lo8) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float y = x[e] * up;
        const _Float16 hi = (_Float16)y, lo = NP == 2 ? (_Float16)(y - (float)hi) : (_Float16)0.f;
        sum += (float)hi + (float)lo;
        const int slot = BITS == 8 ? e : (e % 4) * 2 + e / 4;
        hi8[slot] = hi;
        if constexpr (NP == 2) lo8[slot] = lo;
    }
    return sum;
}

__device__ inline void store_result(const AttendCall &a, int64_t at, float x) {
    if (a.dtype == BIFEAT_F32) static_cast<float *>(a.out)[at] = x;
    else if (a.dtype == BIFEAT_F16) static_cast<Half16 *>(a.out)[at] = from_float<Half16>(x);
    else static_cast<Brain16 *>(a.out)[at] = from_float<Brain16>(x);
}

// four columns of a result row, of which `left` are there
__device__ inline void store_four(const AttendCall &a, int64_t at, int left, const float4 &x) {
    if (a.c.d % 4 == 0 && left >= 4) {
        if (a.dtype == BIFEAT_F32) {
            struct __attribute__((packed, aligned(4))) Four { float4 v; };
            *reinterpret_cast<Four *>(static_cast<float *>(a.out) + at) = Four{x};
        } else {
            struct __attribute__((packed, aligned(2))) Four { uint16_t v[4]; };
            const float e[4] = {x.x, x.y, x.z, x.w};
            Four y;
#pragma unroll
            for (int i = 0; i < 4; i++) y.v[i] = a.dtype == BIFEAT_F16 ? from_float<Half16>(e[i]).bits : from_float<Brain16>(e[i]).bits;
            *reinterpret_cast<Four *>(static_cast<uint16_t *>(a.out) + at) = y;
        }
    } else {
        if (left > 0) store_result(a, at, x.x);
        if (left > 1) store_result(a, at + 1, x.y);
        if (left > 2) store_result(a, at + 2, x.z);
        if (left > 3) store_result(a, at + 3, x.w);
    }
}

// 16 rows of results in LDS, those below `rows`, to where they belong.  A wave.
template <int DP, int STRIDE>
__device__ inline void put_rows(const AttendCall &a, int64_t token0, int head, int row0, int rows, const float *x, int lane) {
    const int64_t heads = (int64_t)a.c.heads * a.group;
    lane = (int)here((uint32_t)lane);
#pragma unroll 1
    for (int i = lane; i < 16 * DP / 4; i += 64) {
        const int r = i / (DP / 4), row = row0 + r, col = i % (DP / 4) * 4;
        if (row >= rows || col >= a.c.d) continue;
        const float4 y = *reinterpret_cast<const float4 *>(x + r * STRIDE + col);
        store_four(a, ((token0 + row / a.group) * heads + head * a.group + row % a.group) * a.c.d + col, a.c.d - col, y);
    }
}

// What a query row sees, as bounds for a position: t <= high and t > low, or t < prefix.
struct Sight {
    int high, low, prefix;
};
__device__ inline Sight sight_of(const AttendCall &a, const View &v, int pos) {
    Sight s;
    s.high = pos < v.len ? pos : v.len - 1;  // (-1 or less for a row that is not there, or lies before the beginning: nothing)
    s.low = a.window && pos >= a.window ? pos - a.window : -1;
    s.prefix = pos >= 0 ? v.prefix : 0;
    return s;
}
// the same of positions at + 0, 1, 2, 3 as four bits
__device__ inline uint32_t seen_of(const Sight &s, int at) {
    uint32_t seen = 0;
#pragma unroll
    for (int t = 0; t < 4; t++) seen |= (uint32_t)((t <= s.high - at && t > s.low - at) || t < s.prefix - at) << t;
    return seen;
}

// cap * tanh(x / cap), both in units of log2.  cap - 2 cap / (e^2u + 1), u = x / cap, is a difference of numbers of the cap's size, off by 2^-23 of
// it however small x is.  For 16-bit results that is enough up to a cap of 64 (2^-17 of a weight, which is rounded to 2^-12).  Otherwise, for
// |u| < 0.6, it is x + x w q(w), w = u^2, with q of degree 3 fitted to (tanh(u) / u - 1) / w (weighted least squares, 2^-23.5 of tanh):
// together within 2^-21 of the result at any cap; a wave whose scores are all below 0.6 of the cap does without the first form.  (First form
// alone and both: 2048 tokens over 8192, cap 30, 128 columns: 546 us and 595; 712 where a wave's scores lie on both sides.)  A
// cap beyond 1e38 is as good as that; one below 1e-37 leaves scores that are as good as 0.
struct Cap {
    float cap, per;  // in units of log2, and 1 / cap
};
__device__ inline Cap cap_of(const AttendCall &a) {
    const float cap = fminf(fmaxf(a.softcap, 1e-37f), 1e38f) * kLog2e;
    return {cap, 1.f / cap};
}
template <bool FIRST, int N>
__device__ inline void cap_all(float (&x)[N], const Cap &c) {
    auto first = [&](float u) { return c.cap - 2.f * c.cap * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(u * (2.f * kLog2e)) + 1.f); };
    if constexpr (FIRST) {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = first(x[i] * c.per);
        return;
    }
    float u[N], most = 0.f;
#pragma unroll
    for (int i = 0; i < N; i++) {
        u[i] = x[i] * c.per;
        most = fmaxf(most, fabsf(u[i]));
        const float w = u[i] * u[i];
        const float q = fmaf(fmaf(fmaf(0.015612629242241383f, w, -0.05221180617809296f), w, 0.13313116133213043f), w, -0.33332598209381104f);
        x[i] = fmaf(x[i] * w, q, x[i]);
    }
    if (__any(!(most < 0.6f)))
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = fabsf(u[i]) < 0.6f ? x[i] : first(u[i]);
}

// p.nw workgroups, in rows: a launch has fewer than 2^32 threads along an axis, 2^24 workgroups
inline dim3 grid_of(const AttendPlan &p) {
    const unsigned x = p.nw < 1 << 23 ? p.nw : 1 << 23;
    return dim3(x, (p.nw + x - 1) / x);
}

void launch_attend_rows(const AttendCall &a, const AttendPlan &p, int bits, int dp);

}  // namespace bf
