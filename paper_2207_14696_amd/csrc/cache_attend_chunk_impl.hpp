// Attention over the paged cache for many query rows a cached head (prompts, chunks of them): 64 NT rows an item.
//
// Bound by vector instructions: a score takes about ten of them (scale and offset of the codes, the exponential at a quarter of
// the rate, two sums, the weight and its rounding), its two products a third of that time on the matrix cores.  So codes become
// operands once a workgroup: each wave makes its share of a tile of TOK positions from registers, where the tile after next
// is on its way, into LDS in the very order in which the products take them (1 KB an operand, 16 bytes a lane, no conflict), and all
// four waves read them there for rows of their own.  Scores are keys x queries as in the kernel for few rows, so that
// weights need not be moved; NT tiles of 16 rows a wave share what is read.
// 2048 tokens over 32 768, 32 heads on 8 of 128 in 8 bits: 1665 us with the join, 640 TFLOP/s; vector instructions are issued 56 % of
// that time, matrix products 28 %.  A batch of 16 prompts and chunks, 12 heads of 64, bias by distance: 329 us, 182 TFLOP/s.
#pragma once

#include "cache_attend.hpp"

namespace bf {

template <int BITS, int DP, int NT>
struct ChunkShape {
    static constexpr int R = 64 * NT, TOK = DP == 256 ? 32 : 64;
    static constexpr int KS = DP / 32, VT = DP / 16;        // operands of 16 keys, of 32 values
    static constexpr int KP = 64 / TOK, VP = 128 / TOK;     // waves that share those
    static constexpr int KB = DP / 4 * BITS / 8 / KP;       // bytes of a key a lane brings
    static constexpr int KL = KB < 16 ? KB : 16;
    static constexpr int VB = DP / 16 * BITS / 8 / VP;      // and of a value
    static constexpr int VW = VB < 4 ? 1 : VB / 4;
    static constexpr int KEYS = TOK / 16 * KS, VALUES = TOK / 32 * VT;
};

// NP: fp16 pieces of a query element and of a weight (2 for 32-bit queries; a second piece of 16-bit results' weights would add to the
// vector instructions, which bound this kernel: fp16 results are off by 3.0e-4 with one, 2.1e-4 of it their own rounding).  MODE: see mode_of
template <int BITS, int DP, int NP, int NT, int MODE>
__global__ __launch_bounds__(256, DP == 256 && NP == 2 ? 1 : 2) void attend_chunk_kernel(AttendCall a, AttendPlan plan) {
    using S = ChunkShape<BITS, DP, NT>;
    constexpr int R = S::R, TOK = S::TOK;
    constexpr float kMiddle = 1 << (BITS - 1);
    extern __shared__ uint4 lds[];
    uint4(*keys)[S::KEYS][64] = reinterpret_cast<uint4(*)[S::KEYS][64]>(lds);
    uint4(*values)[S::VALUES][64] = reinterpret_cast<uint4(*)[S::VALUES][64]>(lds + 2 * S::KEYS * 64);
    float(*params)[4][TOK] = reinterpret_cast<float(*)[4][TOK]>(lds + 2 * (S::KEYS + S::VALUES) * 64);
    __shared__ int sh[16];
    __shared__ float tops[4];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    int cur, end, head;
    Place at;
    locate<R, TOK>(a, plan, (int)blockIdx.x, &cur, &end, &head, &at, sh);

    const int rb = a.c.rb;
    // what this wave brings of a tile: of 16 keys kgroup a quarter of the columns a lane group, of 32 values vgroup
    const int kgroup = wave / S::KP, kpart = wave % S::KP, vgroup = wave / S::VP, vpart = wave % S::VP;
    uint32_t koff[S::KB / S::KL];
#pragma unroll
    for (int i = 0; i < S::KB / S::KL; i++) {
        const int o = (g * S::KP + kpart) * S::KB + i * S::KL;
        koff[i] = n16 * rb + (o < rb ? o : 0);
    }
    const int vo = (n16 * S::VP + vpart) * S::VB;
    const uint32_t voff = 4 * g * rb + (vo < rb ? vo : 0);
    // wave w brings array w of the floats in LDS, a position a lane: key scale times f, key offset (NP == 2: the middle
    // code's value), value scale (1 behind the last position), value of the middle code
    const int fat = lane % TOK;

    while (cur < end) {
        const View v = uniform(view_of<R, TOK>(a, at.seq, at.rt));
        const int units = v.units - at.unit < end - cur ? v.units - at.unit : end - cur;
        const int row0 = at.rt * R, nrows = v.n * a.group - row0 < R ? v.n * a.group - row0 : R;
        const int64_t token0 = uniform(a.b.first(at.seq));

        // ---- pages: lane (TOK / 16) i + j has the page of 16 positions, the j-th of the item's tile `paged` + i
        int pages = 0, paged = -64;
        const int32_t *table = a.b.tables + (int64_t)at.seq * a.b.width;
        constexpr int kSub = TOK / 16;
        // the nearest positions first: with a bias by distance theirs are the largest scores, and sums begun there need not be
        // scaled down tile by tile
        auto base_of = [&](int u) {
            u = at.unit + units - 1 - u;
            return (u < v.skip_at ? u : u + v.skip) * TOK;
        };
        uint32_t kw[S::KB / 4], vw[8][S::VW];
        float fscale, fmin = 0.f;
        auto load = [&](int u) {
            if (u - paged >= 64 / kSub) {
                paged = u;
                int j = u + lane / kSub < units ? base_of(u + lane / kSub) + 16 * (lane % kSub) : 0;
                j = j < v.len ? j : v.len - 1;
                pages = table[j >> a.c.ps_log2];
            }
            const int base = base_of(u), at16 = (u - paged) * kSub;
            auto buffer = [&](int j) { return block_buffer(a.c, __builtin_amdgcn_readlane(pages, at16 + j), head); };
            auto slot = [&](int j) { return (base + 16 * j) & (a.c.ps() - 1); };
            {
                const auto b = buffer(kgroup);
                const uint32_t all = slot(kgroup) * rb;
#pragma unroll
                for (int i = 0; i < S::KB / S::KL; i++) load_bytes<S::KL, false>(b, koff[i], all, &kw[i * S::KL / 4]);
            }
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const auto b = buffer(2 * vgroup + j);
                const uint32_t all = (uint32_t)a.c.codes(1) + slot(2 * vgroup + j) * rb;
#pragma unroll
                for (int i = 0; i < 4; i++) load_bytes<S::VB, false>(b, voff, all + i * rb, vw[4 * j + i]);
            }
            const int page = __shfl(pages, at16 + fat / 16);
            const uint8_t *fp = a.c.block(page, head) + a.c.floats(wave / 2) + 4 * ((base + fat) & (a.c.ps() - 1));
            fscale = *reinterpret_cast<const float *>(fp);
            if (wave & 1) fmin = *reinterpret_cast<const float *>(fp + (4 << a.c.ps_log2));
        };
        float f = 0.f;  // scale of the products, in units of log2
        auto make = [&](int u, int buf) {
#pragma unroll
            for (int c = 0; c < S::KS / S::KP; c++) {
                half8 key;
                if constexpr (BITS == 8) {
                    const uint32_t w0 = kw[2 * c], w1 = kw[2 * c + 1];
                    key = operand(bytes_of(w0, 0), bytes_of(w0, 2), bytes_of(w1, 0), bytes_of(w1, 2));
                } else {
                    key = key_of4(kw[c]);
                }
                if constexpr (NP == 2) key = centred(key, all_of(1152.f));
                keys[buf][kgroup * S::KS + kpart * (S::KS / S::KP) + c][lane] = __builtin_bit_cast(uint4, key);
            }
#pragma unroll
            for (int t = 0; t < S::VT / S::VP; t++) {
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
                values[buf][vgroup * S::VT + vpart * (S::VT / S::VP) + t][lane] = __builtin_bit_cast(uint4, val);
            }
            const bool there = base_of(u) + fat < v.len;  // what no token was written to may hold anything
            float x = there ? fscale : wave == 2 ? 1.f : 0.f;
            if (wave == 0) x *= f;
            if (wave & 1) x = fmaf(x, wave == 3 || NP == 2 ? kMiddle : 0.f, there ? fmin : 0.f);
            if (lane < TOK) params[buf][wave][fat] = x;
        };

        if (v.len > 0) load(0);

        // ---- the queries of the wave's rows
        const int wrow0 = row0 + 16 * NT * wave;  // of the sequence
        const bool any_row = wrow0 < row0 + nrows;
        half8 q[NP][NT][S::KS];
        float qsum[NT], slope[NT];
        int pos[NT];
        {
            // by way of LDS, where no tile is now
            using E = std::conditional_t<NP == 2, float, uint16_t>;
            constexpr int kStride = DP + (NP == 2 && DP != 128 ? 0 : 8);
            E *rows = reinterpret_cast<E *>(lds) + 16 * NT * wave * kStride;
            static_assert(R * kStride * sizeof(E) <= 2 * (S::KEYS + S::VALUES) * 1024, "queries fit the tiles");
            const int at_lane = (int)here((uint32_t)lane);
            const E *own = rows + (at_lane & 15) * kStride + (at_lane >> 4) * (DP / 4);
            if (any_row) stage_queries<16 * NT, DP, kStride>(a, token0, head, wrow0, row0 + nrows, rows, lane, 64);
            wave_sync();
            const bool half = a.dtype == BIFEAT_F16;
            float big = 0.f;
#pragma unroll
            for (int n = 0; n < NT; n++) {
                float its = 0.f;
#pragma unroll
                for (int c = 0; c < S::KS; c++) {
                    float x[8];
                    floats_of(*reinterpret_cast<const Queries8<E> *>(own + 16 * n * kStride + 8 * c), half, x);
                    its = largest_finite(its, x);
                }
                const int row = wrow0 + 16 * n + (at_lane & 15);
                if (v.len - v.n + row / a.group >= 0) big = fmaxf(big, its);
            }
#pragma unroll
            for (int m = 1; m < 64; m *= 2) big = fmaxf(big, __shfl_xor(big, m));
            if (lane == 0) tops[wave] = any_row ? big : 0.f;
            __syncthreads();
            const float up = power_to(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), 14);
            f = a.scale * kLog2e * (kKeyUnit<BITS, NP> / up);
#pragma unroll
            for (int n = 0; n < NT; n++) {
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < S::KS; c++) {
                    float x[8];
                    floats_of(*reinterpret_cast<const Queries8<E> *>(own + 16 * n * kStride + 8 * c), half, x);
                    sum += query_operand<BITS, NP>(x, up, q[0][n][c], q[NP - 1][n][c]);
                }
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                qsum[n] = sum * (f / kKeyUnit<BITS, NP>);
                const int row = wrow0 + 16 * n + (at_lane & 15);
                const bool real = row - row0 < nrows;
                pos[n] = real ? v.len - v.n + row / a.group : -1;
                slope[n] = MODE && a.slopes && real ? a.slopes[head * a.group + row % a.group] * kLog2e : 0.f;
            }
            __syncthreads();
        }
        const Cap cap = cap_of(a);
        // first and last position of the wave's queries
        const int wend = wrow0 + 16 * NT < row0 + nrows ? wrow0 + 16 * NT : row0 + nrows;
        const int wfirst = v.len - v.n + wrow0 / a.group, wlast = v.len - v.n + (wend - 1) / a.group;

        float top[NT], total[NT], mins[NT];  // mins: what is not in the products with the codes
        float4v o[NT][S::VT];
#pragma unroll
        for (int n = 0; n < NT; n++) {
            top[n] = kNothing;
            total[n] = mins[n] = 0.f;
#pragma unroll
            for (int t = 0; t < S::VT; t++) o[n][t] = float4v{0.f, 0.f, 0.f, 0.f};
        }

        // 32 positions for the wave's rows; `whole`: all of them see all
        auto half_tile = [&](bool whole, int base, int buf, int hf) {
            // operands are read ahead of the products that wait for them, as many as there are registers for
            constexpr int kAhead = S::KS < 8 ? S::KS : 4;
            float4v acc[NT][2];
#pragma unroll
            for (int j = 0; j < 2; j++) {
#pragma unroll
                for (int n = 0; n < NT; n++) acc[n][j] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c0 = 0; c0 < S::KS; c0 += kAhead) {
                    half8 key[kAhead];
#pragma unroll
                    for (int c = 0; c < kAhead; c++) key[c] = __builtin_bit_cast(half8, keys[buf][(2 * hf + j) * S::KS + c0 + c][lane]);
#pragma unroll
                    for (int c = 0; c < kAhead; c++)
#pragma unroll
                        for (int p = 0; p < NP; p++)
#pragma unroll
                            for (int n = 0; n < NT; n++)
                                acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key[c], q[p][n][c0 + c], acc[n][j], 0, 0, 0);
                }
            }
            constexpr int kValues = S::VT < 8 ? S::VT : DP * NT > 128 ? 4 : 8;
            half8 val[kValues];
#pragma unroll
            for (int t = 0; t < kValues; t++) val[t] = __builtin_bit_cast(half8, values[buf][hf * S::VT + t][lane]);
            __builtin_amdgcn_sched_barrier(0);
            half8 w[NP][NT];
#pragma unroll
            for (int j = 0; j < 2; j++) {
                float ks[4], km[4], vs[4], vm[4];
                {
                    float4 x[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) x[i] = *reinterpret_cast<const float4 *>(&params[buf][i][32 * hf + 16 * j + 4 * g]);
#pragma unroll
                    for (int i = 0; i < 4; i++) ks[i] = (&x[0].x)[i], km[i] = (&x[1].x)[i], vs[i] = (&x[2].x)[i], vm[i] = (&x[3].x)[i];
                }
                const int at4 = base + 16 * j + 4 * g;
                uint32_t seen[NT];
#pragma unroll
                for (int n = 0; n < NT; n++) seen[n] = whole ? 15u : seen_of(sight_of(a, v, pos[n]), at4);
                float p[NT][4], pw[NT][4];
                // scores less `ref`, -infinity where the row does not see the position
                auto score = [&](int n, float ref, float(&y)[4]) {
                    if constexpr (MODE == kPlain) {
#pragma unroll
                        for (int i = 0; i < 4; i++) y[i] = fmaf(ks[i], acc[n][j][i], fmaf(km[i], qsum[n], -ref));
                    } else if constexpr (MODE == kBiased) {
                        const float from = fmaf(slope[n], (float)(at4 - pos[n]), -ref);
#pragma unroll
                        for (int i = 0; i < 4; i++) y[i] = fmaf(ks[i], acc[n][j][i], fmaf(km[i], qsum[n], fmaf(slope[n], (float)i, from)));
                    } else {
                        const float from = fmaf(slope[n], (float)(at4 - pos[n]), -ref);
#pragma unroll
                        for (int i = 0; i < 4; i++) y[i] = fmaf(ks[i], acc[n][j][i], km[i] * qsum[n]);
                        cap_all<MODE == kCappedFirst>(y, cap);
#pragma unroll
                        for (int i = 0; i < 4; i++) y[i] += fmaf(slope[n], (float)i, from);
                    }
                    if (!whole) {
                        const uint32_t bits = here(seen[n]);
#pragma unroll
                        for (int i = 0; i < 4; i++) y[i] = bits >> i & 1 ? y[i] : -INFINITY;
                    }
                };
                // infinite where a value's size (see size_of) is not its scale.  (2 % of 2048 tokens over 32 768, as much as a flag a tile)
                const float sized = fminf(fminf(vs[0], vs[1]), fminf(vs[2], vs[3])) < kLeastScale ? INFINITY : 0.f;
                auto weigh = [&] {
                    float most = sized;
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        float y[4];
                        score(n, top[n], y);
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            p[n][i] = __builtin_amdgcn_exp2f(y[i]);
                            pw[n][i] = p[n][i] * vs[i];
                            most = fmaxf(most, pw[n][i]);
                        }
                    }
                    return most;
                };
                if (__any(weigh() > 32768.f)) {
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        float y[4], now = kNothing;
                        score(n, 0.f, y);
#pragma unroll
                        for (int i = 0; i < 4; i++) now = fmaxf(now, y[i] + __builtin_amdgcn_logf(size_of(vs[i], vm[i])));
                        now = fmaxf(now, __shfl_xor(now, 16));
                        now = fmaxf(now, __shfl_xor(now, 32));
                        now = fmaxf(top[n], ceilf(now) - 8.f);  // (whole numbers: what is kept is kept exactly)
                        const float keep = __builtin_amdgcn_exp2f(top[n] - now);
                        top[n] = now;
                        total[n] *= keep;
                        mins[n] *= keep;
#pragma unroll
                        for (int t = 0; t < S::VT; t++) o[n][t] *= keep;
                        if (j)
#pragma unroll
                            for (int k = 0; k < NP; k++)
#pragma unroll
                                for (int i = 0; i < 4; i++) w[k][n][i] *= (_Float16)keep;
                    }
                    weigh();
                }
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 4; i++) mins[n] = fmaf(p[n][i], vm[i], mins[n]);
                    } else {  // (an infinity or NaN that the row does not see is not to reach it)
                        const uint32_t bits = here(seen[n]);
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            mins[n] = bits >> i & 1 ? fmaf(p[n][i], vm[i], mins[n]) : mins[n];
                            pw[n][i] = bits >> i & 1 ? pw[n][i] : 0.f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        total[n] += p[n][i];
                        w[0][n][4 * j + i] = (_Float16)pw[n][i];
                        if constexpr (NP == 2) w[NP - 1][n][4 * j + i] = (_Float16)(pw[n][i] - (float)w[0][n][4 * j + i]);
                    }
                    if constexpr (NP == 1)
#pragma unroll
                        for (int i = 4 * j; i < 4 * j + 4; i += 2)
                            mins[n] = __builtin_amdgcn_fdot2(half2v{w[0][n][i], w[0][n][i + 1]}, half2v{(_Float16)-kMiddle, (_Float16)-kMiddle}, mins[n], false);
                }
            }
#pragma unroll
            for (int t = 0; t < S::VT; t++) {
                if (t >= kValues) val[t % kValues] = __builtin_bit_cast(half8, values[buf][hf * S::VT + t][lane]);
#pragma unroll
                for (int p = 0; p < NP; p++)
#pragma unroll
                    for (int n = 0; n < NT; n++)
                        o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(val[t % kValues], w[p][n], o[n][t], 0, 0, 0);
            }
        };

        if (v.len > 0) {
            make(0, 0);
            if (units > 1) load(1);
            __syncthreads();
            for (int u = 0; u < units; u++) {
                const int base = base_of(u), buf = u & 1;
                if (u + 1 < units) make(u + 1, buf ^ 1);
                if (u + 2 < units) load(u + 2);
                if (any_row)
#pragma unroll 1
                    for (int hf = 0; hf < TOK / 32; hf++) {
                        const int b = base + 32 * hf;
                        // positions that none of the wave's rows sees
                        if (b >= v.len || ((b > wlast || (a.window && b + 31 <= wfirst - a.window)) && b >= v.prefix)) continue;
                        // do all rows see all of them?
                        const bool whole = b + 32 <= v.len && wfirst >= 0 &&
                                           ((b + 31 <= wfirst && (!a.window || b > wlast - a.window)) || b + 32 <= v.prefix);
                        half_tile(whole, b, buf, hf);
                    }
                __syncthreads();
            }
        }

        const bool complete = at.unit == 0 && units == v.units;
        constexpr int kOut = DP + 4;
        static_assert(4 * 16 * kOut * sizeof(float) <= 2 * (S::KEYS + S::VALUES) * 1024 + 8 * TOK * sizeof(float), "a tile of rows a wave fits");
        if (any_row) {
            const int at_lane = (int)here((uint32_t)lane), row16 = at_lane & 15, quarter = at_lane >> 4;
#pragma unroll
            for (int n = 0; n < NT; n++) {
                float s = total[n], rest = mins[n];
                s += __shfl_xor(s, 16);
                s += __shfl_xor(s, 32);
                rest += __shfl_xor(rest, 16);
                rest += __shfl_xor(rest, 32);
                // by way of LDS, where the tiles are done with, to rows of consecutive columns
                const float inv = complete ? (s != 0.f ? 1.f / s : 0.f) : 1.f;
                float *x = reinterpret_cast<float *>(lds) + wave * 16 * kOut;
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int t = 0; t < S::VT; t++)
                        x[row16 * kOut + (4 * quarter + i) * S::VT + t] =
                            fmaf(o[n][t][i], kUnit<NP> * (BITS == 4 && (t & 1) ? 0.0625f : 1.f), rest) * inv;
                wave_sync();
                const int r0 = 16 * (NT * wave + n);
                if (complete) {
                    put_rows<DP, kOut>(a, token0, head, row0 + r0, row0 + nrows, x, lane);
                } else {
                    float *part = plan.partial + ((int64_t)blockIdx.x * 2 + (at.unit == 0)) * (R * (DP + 2));
                    if (quarter == 0) part[R * DP + r0 + row16] = top[n], part[R * DP + R + r0 + row16] = s;
#pragma unroll 1
                    for (int i = at_lane; i < 16 * DP / 4; i += 64)
                        *reinterpret_cast<float4 *>(part + r0 * DP + 4 * i) = *reinterpret_cast<const float4 *>(x + i / (DP / 4) * kOut + i % (DP / 4) * 4);
                }
                wave_sync();
            }
        }
        __syncthreads();
        cur += units;
        if (cur < end) next_item<R>(a, &head, &at);
    }
}

template <int BITS, int DP, int NT>
constexpr size_t chunk_lds() {
    using S = ChunkShape<BITS, DP, NT>;
    return 2 * ((S::KEYS + S::VALUES) * 1024 + 4 * S::TOK * sizeof(float));
}

}  // namespace bf
