// Attention over the paged cache for few query rows a cached head (single tokens, a few drafted ones): 16 rows an item.
//
// Bound by the cache's bytes: a cached row is fetched once for all query heads that share it.  Everything stays in
// registers.  A wave takes 32 positions a step, the four waves of a workgroup every fourth step; a step's keys make room
// for the next one's as soon as the scores are there, its values when the sums are, so that one or the other is always on
// its way.  Scores are keys x queries (positions the rows of the 16 x 16 product), so that a lane ends up with
// four positions of one query, which is how the second product wants its weights: nothing is moved between lanes.
// 64 single tokens over up to 8192 positions, 32 heads on 8 of 128 in 8 bits (622 MB): 119 us, 5.2 TB/s; four over 131 072, 64 heads on 8,
// 4 bits (604 MB): 116, 5.2 TB/s.  Of its waves' time 40 to 44 % waits for memory, 17 to 29 % issues vector instructions.
#pragma once

#include "cache_attend.hpp"

namespace bf {

template <int BITS, int DP>
struct RowLanes {
    static constexpr int KB = DP / 4 * BITS / 8;   // bytes of a key that a lane reads (its quarter of the columns)
    static constexpr int KL = KB < 16 ? KB : 16;   // in loads of so many, four lanes' next to each other
    static constexpr int KC = KL * 8 / BITS;       // columns a load
    static constexpr int VB = DP / 16 * BITS / 8;  // bytes of a value (its sixteenth)
    static constexpr int KS = DP / 32;             // products over the columns
    static constexpr int VT = DP / 16;             // tiles of the values' columns
    static constexpr int VW = VB < 4 ? 1 : VB / 4;
};

// NP: fp16 pieces of a query element (2 for 32-bit queries); WP: of a weight.  One is enough where the result is rounded to
// bf16 (2^-9; a weight's one piece 2^-12, the second costs 8 % of long contexts in 4 bits); an fp16 result would be 1.6 times as far off
// with one, and the second costs it 1 %.  MODE: see mode_of.
template <int BITS, int DP, int NP, int WP, int MODE>
__global__ __launch_bounds__(256, DP == 256 ? 1 : DP == 128 ? 2 : 3) void attend_rows_kernel(AttendCall a, AttendPlan plan) {
    using L = RowLanes<BITS, DP>;
    constexpr int R = kRowsR, TOK = kRowsTok;
    constexpr float kMiddle = 1 << (BITS - 1);
    __shared__ float sums[4][R][DP + 4];
    __shared__ float tops[4][R], totals[4][R];
    __shared__ float params[4][4][32];  // a wave's step: key scale, key minimum, value scale, value minimum
    __shared__ int sh[16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    int cur, end, head;
    Place at;
    locate<R, TOK>(a, plan, (int)blockIdx.x, &cur, &end, &head, &at, sh);

    // byte offsets in a row; past its end (columns the row is too short for) any byte will do: the queries have zeros there,
    // and the sums of such columns are not written
    const int rb = a.c.rb;
    uint32_t koff[L::KB / L::KL];
#pragma unroll
    for (int i = 0; i < L::KB / L::KL; i++) {
        const int o = (4 * i + g) * L::KL;
        koff[i] = n16 * rb + (o < rb ? o : 0);
    }
    const uint32_t voff = 4 * g * rb + (n16 * L::VB < rb ? n16 * L::VB : 0);
    // lane l < 32 brings four positions' worth of one of the four floats
    const uint32_t foff = ((lane >> 3 & 3) * 4u << a.c.ps_log2) + 16 * (lane & 3);

    while (cur < end) {
        const View v = uniform(view_of<R, TOK>(a, at.seq, at.rt));
        const int units = v.units - at.unit < end - cur ? v.units - at.unit : end - cur;
        const int row0 = at.rt * R, nrows = v.n * a.group - row0 < R ? v.n * a.group - row0 : R;
        const int64_t token0 = uniform(a.b.first(at.seq));

        // ---- pages: lane 2 i + j has the page of the wave's i-th step from `paged` on, half j
        int pages = 0, paged = -64;
        const int32_t *table = a.b.tables + (int64_t)at.seq * a.b.width;
        auto base_of = [&](int u) {  // first position of the wave's step in unit u of the item
            u = at.unit + units - 1 - u;  // the nearest first
            return (u < v.skip_at ? u : u + v.skip) * TOK + 32 * wave;
        };
        uint32_t kw[2][L::KB / 4], vw[8][L::VW];
        float4 fw;
        __amdgpu_buffer_rsrc_t block0, block1;  // of the step's two halves
        int slot0, slot1;
        // Asked for without a branch, of no block where the item has no such unit: across a branch the compiler could not tell how
        // many loads are on their way, and would wait for all of them where it needs the oldest (contexts of 131 072 tokens in 4
        // bits 121 us, 117 so).  Past the caches: 64 single tokens over up to 8192 130 us, 119 so; also where items share what they read, which is
        // slower for caches that would hold it (64 rows of 8 sequences of 2048 34.7 us, 38.0 so; 32 x 5 tokens of 256 columns 44.2 and 47.2) and
        // faster for larger ones (64 rows of 64 of 4096, 12 heads of 64: 321 and 289).
        auto load_keys = [&](int u) {
            const bool wanted = u < units;
            if (wanted && u - paged >= 32) {
                paged = u;
                int j = u + (lane >> 1) < units ? base_of(u + (lane >> 1)) + 16 * (lane & 1) : 0;
                j = j < v.len ? j : v.len - 1;
                pages = table[j >> a.c.ps_log2];
            }
            const int page0 = __builtin_amdgcn_readlane(pages, 2 * (u - paged) & 63), page1 = __builtin_amdgcn_readlane(pages, (2 * (u - paged) & 63) + 1);
            block0 = block_buffer(a.c, page0, head, wanted);
            block1 = block_buffer(a.c, page1, head, wanted);
            slot0 = base_of(u) & (a.c.ps() - 1);
            slot1 = (base_of(u) + 16) & (a.c.ps() - 1);
#pragma unroll
            for (int i = 0; i < L::KB / L::KL; i++) load_bytes<L::KL, true>(block0, koff[i], slot0 * rb, &kw[0][i * L::KL / 4]);
#pragma unroll
            for (int i = 0; i < L::KB / L::KL; i++) load_bytes<L::KL, true>(block1, koff[i], slot1 * rb, &kw[1][i * L::KL / 4]);
            const uint8_t *fp = a.c.block(lane & 4 ? page1 : page0, head) + a.c.floats(0) + 4 * (lane & 4 ? slot1 : slot0);
            fw = *reinterpret_cast<const float4 *>(fp + foff);
        };
        auto load_values = [&] {  // of the step whose keys were asked for last
            const uint32_t at0 = (uint32_t)a.c.codes(1) + slot0 * rb, at1 = (uint32_t)a.c.codes(1) + slot1 * rb;
#pragma unroll
            for (int i = 0; i < 4; i++) load_bytes<L::VB, true>(block0, voff, at0 + i * rb, vw[i]);
#pragma unroll
            for (int i = 0; i < 4; i++) load_bytes<L::VB, true>(block1, voff, at1 + i * rb, vw[4 + i]);
        };

        if (v.len > 0) {
            load_keys(0);
            load_values();
        }

        // ---- the queries: lane (n16, g) has a quarter of the columns of row n16, those of the keys that it reads
        const int row = row0 + n16;
        const bool real = n16 < nrows;
        const int qi = row / a.group, qh = head * a.group + row % a.group;
        const int pos = real ? v.len - v.n + qi : -1;
        half8 q[NP][L::KS];
        float qsum = 0.f, f;
        {
            using E = std::conditional_t<NP == 2, float, uint16_t>;
            constexpr int kStride = DP + 8;
            Queries8<E> raw[L::KS];  // the columns of the c-th 8 codes of this lane's keys
            const int at_lane = (int)here((uint32_t)lane);
            auto column = [&](int c) { return (4 * (8 * c / L::KC) + (at_lane >> 4)) * L::KC + 8 * c % L::KC; };
            if (a.c.d % 4 == 0) {
                const int r = real ? row : row0;
                const E *q = static_cast<const E *>(a.q.data) + (token0 + r / a.group) * a.q.token_stride +
                             ((int64_t)head * a.group + r % a.group) * a.q.head_stride;
                struct __attribute__((packed, aligned(sizeof(E)))) Four { E v[4]; };
#pragma unroll
                for (int c = 0; c < L::KS; c++)
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        const bool there = real && column(c) + h < a.c.d;
                        const Four y = *reinterpret_cast<const Four *>(q + (there ? column(c) + h : 0));
#pragma unroll
                        for (int e = 0; e < 4; e++) raw[c].v[h + e] = there ? y.v[e] : (E)0;
                    }
            } else {  // by way of LDS, where nothing is summed now
                E *rows = reinterpret_cast<E *>(&sums[0][0][0]);
                stage_queries<R, DP, kStride>(a, token0, head, row0, row0 + nrows, rows, threadIdx.x, 256);
                __syncthreads();
#pragma unroll
                for (int c = 0; c < L::KS; c++) raw[c] = *reinterpret_cast<const Queries8<E> *>(rows + (at_lane & 15) * kStride + column(c));
                __syncthreads();
            }
            const bool half = a.dtype == BIFEAT_F16;
            float big = 0.f;
#pragma unroll
            for (int c = 0; c < L::KS; c++) {
                float x[8];
                floats_of(raw[c], half, x);
                big = largest_finite(big, x);
            }
            if (pos < 0) big = 0.f;
#pragma unroll
            for (int m = 1; m < 64; m *= 2) big = fmaxf(big, __shfl_xor(big, m));
            const float up = power_to(big, 14);
            f = a.scale * kLog2e * (kKeyUnit<BITS, NP> / up);
#pragma unroll
            for (int c = 0; c < L::KS; c++) {
                float x[8];
                floats_of(raw[c], half, x);
                qsum += query_operand<BITS, NP>(x, up, q[0][c], q[NP - 1][c]);
            }
            qsum += __shfl_xor(qsum, 16);
            qsum += __shfl_xor(qsum, 32);
            qsum *= f / kKeyUnit<BITS, NP>;
        }
        const float slope = MODE && a.slopes ? a.slopes[real ? qh : 0] * kLog2e : 0.f;
        const Cap cap = cap_of(a);

        float top = kNothing, total = 0.f, mins = 0.f;  // mins: what is not in the products with the codes
        float4v o[L::VT];
#pragma unroll
        for (int t = 0; t < L::VT; t++) o[t] = float4v{0.f, 0.f, 0.f, 0.f};

        auto step = [&](bool whole, int base, int next) {
            const bool sized = __any((lane >> 3 & 3) == 2 && fminf(fminf(fw.x, fw.y), fminf(fw.z, fw.w)) < kLeastScale);  // (see size_of)
            wave_sync();
            if (lane < 32) *reinterpret_cast<float4 *>(&params[wave][lane >> 3][4 * (lane & 7)]) = fw;
            wave_sync();
            float ks[8], km[8], vs[8], vm[8];
#pragma unroll
            for (int j = 0; j < 2; j++) {
                float4 p[4];
#pragma unroll
                for (int i = 0; i < 4; i++) p[i] = *reinterpret_cast<const float4 *>(&params[wave][i][16 * j + 4 * g]);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int e = 4 * j + i;
                    ks[e] = (&p[0].x)[i];
                    km[e] = NP == 2 ? fmaf(ks[e], kMiddle, (&p[1].x)[i]) : (&p[1].x)[i];
                    vs[e] = (&p[2].x)[i];
                    vm[e] = fmaf(vs[e], kMiddle, (&p[3].x)[i]);
                }
            }
            uint32_t seen = 0xffu;
            if (!whole) {
                const Sight sight = sight_of(a, v, pos);
                seen = seen_of(sight, base + 4 * g) | seen_of(sight, base + 16 + 4 * g) << 4;
            }
            // ---- scores
            float4v acc[2];
#pragma unroll
            for (int j = 0; j < 2; j++) {
                acc[j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < L::KS; c++) {
                    half8 key;
                    if constexpr (BITS == 8) {
                        const uint32_t w0 = kw[j][2 * c], w1 = kw[j][2 * c + 1];
                        key = operand(bytes_of(w0, 0), bytes_of(w0, 2), bytes_of(w1, 0), bytes_of(w1, 2));
                    } else {
                        key = key_of4(kw[j][c]);
                    }
                    if constexpr (NP == 2) key = centred(key, all_of(1152.f));
#pragma unroll
                    for (int p = 0; p < NP; p++) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key, q[p][c], acc[j], 0, 0, 0);
                }
            }
            load_keys(next);
            float p[8], pw[8], y[8];
            // scores less `ref`, -infinity where the row does not see the position
            auto score = [&](float ref) {
                const float from = MODE ? fmaf(slope, (float)(base + 4 * g - pos), -ref) : -ref;
                if constexpr (MODE >= kCappedFirst) {
#pragma unroll
                    for (int e = 0; e < 8; e++) y[e] = fmaf(ks[e], f * acc[e / 4][e % 4], km[e] * qsum);
                    cap_all<MODE == kCappedFirst>(y, cap);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float bias = MODE ? fmaf(slope, (float)(16 * (e / 4) + e % 4), from) : from;
                    if constexpr (MODE < kCappedFirst) y[e] = fmaf(ks[e], f * acc[e / 4][e % 4], fmaf(km[e], qsum, bias));
                    else y[e] += bias;
                }
                if (!whole) {
                    const uint32_t bits = here(seen);
#pragma unroll
                    for (int e = 0; e < 8; e++) y[e] = bits >> e & 1 ? y[e] : -INFINITY;
                }
            };
            auto weigh = [&] {
                float most = 0.f;
                score(top);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    p[e] = __builtin_amdgcn_exp2f(y[e]);
                    pw[e] = p[e] * vs[e];
                    most = fmaxf(most, pw[e]);
                }
                return most;
            };
            if (__any(weigh() > 32768.f) || sized) {
                float now = kNothing;
                score(0.f);
#pragma unroll
                for (int e = 0; e < 8; e++) now = fmaxf(now, y[e] + __builtin_amdgcn_logf(size_of(vs[e], vm[e])));
                now = fmaxf(now, __shfl_xor(now, 16));
                now = fmaxf(now, __shfl_xor(now, 32));
                now = fmaxf(top, ceilf(now) - 8.f);  // (whole numbers: what is kept is kept exactly)
                const float keep = __builtin_amdgcn_exp2f(top - now);
                top = now;
                total *= keep;
                mins *= keep;
#pragma unroll
                for (int t = 0; t < L::VT; t++) o[t] *= keep;
                weigh();
            }
            // ---- weights
            half8 w[WP];
            if (whole) {
#pragma unroll
                for (int e = 0; e < 8; e++) mins = fmaf(p[e], vm[e], mins);
            } else {  // (an infinity or NaN that the row does not see is not to reach it)
                const uint32_t bits = here(seen);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    mins = bits >> e & 1 ? fmaf(p[e], vm[e], mins) : mins;
                    pw[e] = bits >> e & 1 ? pw[e] : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                total += p[e];
                w[0][e] = (_Float16)pw[e];
                if constexpr (WP == 2) w[WP - 1][e] = (_Float16)(pw[e] - (float)w[0][e]);
            }
            if constexpr (NP == 1)
#pragma unroll
                for (int p = 0; p < WP; p++)
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        mins = __builtin_amdgcn_fdot2(half2v{w[p][e], w[p][e + 1]}, half2v{(_Float16)-kMiddle, (_Float16)-kMiddle}, mins, false);
            // ---- values: lane (n16, g) has columns [n16 DP/16, ...) of eight positions
#pragma unroll
            for (int t = 0; t < L::VT; t++) {
                half8 val;
                if constexpr (BITS == 8) {
                    val = operand(pair_of(vw[0][t / 4], vw[1][t / 4], t % 4), pair_of(vw[2][t / 4], vw[3][t / 4], t % 4),
                                  pair_of(vw[4][t / 4], vw[5][t / 4], t % 4), pair_of(vw[6][t / 4], vw[7][t / 4], t % 4));
                } else {
                    const int i = t / 2 % 4, d = t / 8;
                    const uint32_t mask = t & 1 ? 0x00f000f0u : 0x000f000fu;
                    val = operand(pair_of(vw[0][d], vw[1][d], i) & mask, pair_of(vw[2][d], vw[3][d], i) & mask,
                                  pair_of(vw[4][d], vw[5][d], i) & mask, pair_of(vw[6][d], vw[7][d], i) & mask);
                }
                if constexpr (NP == 2) val = centred(val, all_of(BITS == 8 || (t & 1) ? 1152.f : 1032.f));
#pragma unroll
                for (int p = 0; p < WP; p++)
                    o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(val, w[p], o[t], 0, 0, 0);
            }
        };

        if (v.len > 0)
            for (int u = 0; u < units; u++) {
                const int base = base_of(u);
                if (base < v.len) {  // (of the context's last positions some waves may have none)
                    // do all rows see all 32 positions?
                    const bool whole = base + 32 <= v.len && v.first >= 0 &&
                                       ((base + 31 <= v.first && (!a.window || base > v.last - a.window)) || base + 32 <= v.prefix);
                    step(whole, base, u + 1);
                } else {
                    load_keys(u + 1);
                }
                load_values();
            }

        // ---- the four waves' parts joined
        const int at_lane = (int)here((uint32_t)lane), row16 = at_lane & 15, quarter = at_lane >> 4;
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
        mins += __shfl_xor(mins, 16);
        mins += __shfl_xor(mins, 32);
#pragma unroll
        for (int t = 0; t < L::VT; t++) {
            const float back = kUnit<NP> * (BITS == 4 && (t & 1) ? 0.0625f : 1.f);
#pragma unroll
            for (int i = 0; i < 4; i++) sums[wave][row16][(4 * quarter + i) * L::VT + t] = fmaf(o[t][i], back, mins);
        }
        if (quarter == 0) {
            tops[wave][row16] = top;
            totals[wave][row16] = total;
        }
        __syncthreads();
        {
            const int me = (int)here(threadIdx.x), r = me >> 4, c0 = me & 15;
            const float t0 = tops[0][r], t1 = tops[1][r], t2 = tops[2][r], t3 = tops[3][r];
            const float now = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3));
            const float e0 = __builtin_amdgcn_exp2f(t0 - now), e1 = __builtin_amdgcn_exp2f(t1 - now);
            const float e2 = __builtin_amdgcn_exp2f(t2 - now), e3 = __builtin_amdgcn_exp2f(t3 - now);
            const float all = totals[0][r] * e0 + totals[1][r] * e1 + totals[2][r] * e2 + totals[3][r] * e3;
            const bool whole = at.unit == 0 && units == v.units;
            float *part = whole ? nullptr : plan.partial + ((int64_t)blockIdx.x * 2 + (at.unit == 0)) * (R * (DP + 2));
            const int64_t dst = ((token0 + (row0 + r) / a.group) * ((int64_t)a.c.heads * a.group) + head * a.group + (row0 + r) % a.group) * a.c.d;
            const float inv = all != 0.f ? 1.f / all : 0.f;
            if (r < nrows) {
                for (int c = c0; c < a.c.d; c += 16) {
                    const float x = sums[0][r][c] * e0 + sums[1][r][c] * e1 + sums[2][r][c] * e2 + sums[3][r][c] * e3;
                    if (whole) store_result(a, dst + c, x * inv);
                    else part[r * DP + c] = x;
                }
                if (!whole && c0 == 0) part[R * DP + r] = now, part[R * DP + R + r] = all;
            }
        }
        __syncthreads();
        cur += units;
        if (cur < end) next_item<R>(a, &head, &at);
    }
}

}  // namespace bf
