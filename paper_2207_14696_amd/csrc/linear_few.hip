// Products of few rows with matrices in 4 bits.
#include <algorithm>

#include "linear.hpp"

namespace bf {
namespace {

// A workgroup takes R times 16 rows of the matrix, up to 16 TB rows of x and, where the columns are split, a part of these; its waves take blocks of 128 columns in turn and add up what they have
// in LDS at the end.  A lane's 16 bytes of a block are 32 codes of one row of the matrix, four operands as they are; x is the other operand, so that a lane's sums
// are of one row of the matrix, and of one scale.  Of up to 16 rows the next block
// is on its way while one is multiplied.
template <typename T, int GPB, int TB, int R, int kWaves, bool DEALT, typename Out>
__global__ __launch_bounds__(64 * kWaves) void linear_few_kernel(Matrices m, XRows x, Deal deal, Out *out, int tile0) {
    typedef Operand<T> O;
    constexpr int P = O::kPieces;
    __shared__ Sum4 part[kWaves][R * TB][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quarter = lane / 16;
    const int row0 = blockIdx.x * R;
    const int x_tile = tile0 + blockIdx.y;
    const int64_t first = (int64_t)x_tile * 16 * TB;
    int count;
    const uint8_t *packed = m.packed;
    // the tile's rows: what a lane brings, and the four that it stores
    const int mine[4] = {4 * quarter, 4 * quarter + 1, 4 * quarter + 2, 4 * quarter + 3};
    int64_t from[TB], to[4];
    if constexpr (DEALT) {
        // (all of it asked for at a time; places that are not filled are the first one's)
        const int tiles = *deal.tiles_count;
        const Tile t = deal.tiles[x_tile];
        const int head = deal.order[first];
        int mine_to[4], mine_from = deal.order[first + col];
#pragma unroll
        for (int j = 0; j < 4; j++) mine_to[j] = deal.order[first + mine[j]];
        if (x_tile >= tiles) return;
        count = t.count;
        if (t.expert < 0) {
            for (int i = threadIdx.x; i < count * 16 * R; i += 64 * kWaves) {
                const int n = 16 * row0 + i % (16 * R);
                if (n < m.N) out[(int64_t)deal.order[first + i / (16 * R)] * m.N + n] = from_float<Out>(0.f);
            }
            return;
        }
        packed += t.expert * m.bytes;
        from[0] = col < count ? mine_from : head;
#pragma unroll
        for (int j = 0; j < 4; j++) to[j] = mine_to[j];
    } else {
        count = x.count - first < 16 * TB ? (int)(x.count - first) : 16 * TB;
#pragma unroll
        for (int t = 0; t < TB; t++) from[t] = first + (16 * t + col < count ? 16 * t + col : count - 1);  // (what a row past the last gives is not stored)
    }
    const T *xr[TB];
#pragma unroll
    for (int t = 0; t < TB; t++) {
        const int64_t row = from[t], token = DEALT ? (int64_t)((uint32_t)row / (uint32_t)x.choices) : row;
        xr[t] = static_cast<const T *>(x.x) + token * x.token_stride + (DEALT ? (row - token * x.choices) * x.choice_stride : 0);
    }
    // the part of the columns, in blocks
    const int begin = (int)((int64_t)m.blocks * blockIdx.z / gridDim.z), end = (int)((int64_t)m.blocks * (blockIdx.z + 1) / gridDim.z);
    if constexpr (!DEALT) out += blockIdx.z * x.count * m.N;
    const uint4 *codes[R];
    const uint32_t *levels[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t at = (int64_t)(row0 + r < m.rows ? row0 + r : m.rows - 1) * m.blocks;
        codes[r] = reinterpret_cast<const uint4 *>(packed) + at * 64 + lane;
        levels[r] = reinterpret_cast<const uint32_t *>(packed + m.code_bytes()) + at * GPB * 16 + col;
    }
    Sum4 total[R][TB];
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int t = 0; t < TB; t++) total[r][t] = 0.f;
    struct Block {
        uint4 codes[R];
        uint32_t level[R][GPB];
        Columns<T> columns[4][TB];
    };
    const auto bring_matrix = [&](Block &b, int k) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            b.codes[r] = codes[r][(int64_t)k * 64];
#pragma unroll
            for (int g = 0; g < GPB; g++) b.level[r][g] = levels[r][(k * GPB + g) * 16];
        }
    };
    const auto bring_rows = [&](Block &b, int k, auto of) {
#pragma unroll
        for (int w = 0; w < 4; w++)
#pragma unroll
            for (int t = 0; t < TB; t++) b.columns[w][t] = of(xr[t], 128 * k + 32 * w + 8 * quarter);
    };
    const auto multiply = [&](const Block &b) {
#pragma unroll
        for (int g = 0; g < GPB; g++) {
            Sum4 sum[R][TB], of_x[TB];
#pragma unroll
            for (int t = 0; t < TB; t++) {
                of_x[t] = 0.f;
#pragma unroll
                for (int r = 0; r < R; r++) sum[r][t] = 0.f;
            }
#pragma unroll
            for (int w = 4 / GPB * g; w < 4 / GPB * (g + 1); w++) {
                typename O::Eight c[R], o[TB][P];
#pragma unroll
                for (int t = 0; t < TB; t++) to_operands<T>(b.columns[w][t], o[t]);
#pragma unroll
                for (int r = 0; r < R; r++) c[r] = code_operands<T>(w == 0 ? b.codes[r].x : w == 1 ? b.codes[r].y : w == 2 ? b.codes[r].z : b.codes[r].w);
#pragma unroll
                for (int t = 0; t < TB; t++)
#pragma unroll
                    for (int p = 0; p < P; p++) {
                        of_x[t] = O::product(o[t][p], ones<T>(), of_x[t]);
#pragma unroll
                        for (int r = 0; r < R; r++) sum[r][t] = O::product(o[t][p], c[r], sum[r][t]);
                    }
            }
#pragma unroll
            for (int r = 0; r < R; r++) {
                const float scale = __builtin_bit_cast(float, b.level[r][g] << 16), low = __builtin_bit_cast(float, b.level[r][g] & 0xffff0000u);
                const float rest = fmaf(-O::kMore, scale, low);
#pragma unroll
                for (int t = 0; t < TB; t++)
#pragma unroll
                    for (int i = 0; i < 4; i++) total[r][t][i] = fmaf(scale, sum[r][t][i], fmaf(rest, of_x[t][i], total[r][t][i]));
            }
            if constexpr (TB * R >= 12) {  // (here and not where they are used next: the compiler would keep what they are made of until then)
#pragma unroll
                for (int r = 0; r < R; r++)
#pragma unroll
                    for (int t = 0; t < TB; t++) asm volatile("" : "+v"(total[r][t]));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    const auto whole = [](const T *row, int at) { return load_columns(row + at); };
    const int full = m.K / 128 < end ? m.K / 128 : end;
    int k = begin + wave;
    Block now;
    if (TB == 1 && k < full) {
        bring_matrix(now, k);
        bring_rows(now, k, whole);
    }
    for (; k < full; k += kWaves) {
        if constexpr (TB == 1) {
            Block next;
            if (k + kWaves < full) {
                bring_matrix(next, k + kWaves);
                bring_rows(next, k + kWaves, whole);
            }
            multiply(now);
            now = next;
        } else {
            bring_matrix(now, k);
            bring_rows(now, k, whole);
            multiply(now);
        }
    }
    if (full < end && wave == (full - begin) % kWaves) {
        Block last;
        bring_matrix(last, full);
        if (m.K >= 8) bring_rows(last, full, [&](const T *row, int at) { return load_last_columns(row, at, m.K); });
        else bring_rows(last, full, [&](const T *row, int at) { return at == 0 ? load_short_columns(row, m.K) : no_columns<T>(); });
        multiply(last);
    }
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int t = 0; t < TB; t++) part[wave][r * TB + t][lane] = total[r][t];
    __syncthreads();
    for (int i = wave; i < R * TB; i += kWaves) {
        Sum4 y = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < kWaves; w++) y += part[w][i][lane];
        const int r = i / TB, t = i - r * TB, n = 16 * (row0 + r) + col;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int at = 16 * t + mine[j];
            if (at < count && n < m.N) out[(DEALT ? to[j] : first + at) * m.N + n] = from_float<Out>(y[j]);
        }
    }
}

template <typename T, typename Out, bool DEALT>
void go(const Matrices &m, int group, const XRows &x, const Deal &deal, int64_t tiles, const FewShape &shape, hipStream_t s) {
    const auto launch = [&](auto kernel, int tb, int r, int waves) {
        const int64_t y = DEALT ? tiles : (x.count + 16 * tb - 1) / (16 * tb);
        const int row_tiles = (m.rows + r - 1) / r;
        // (a launch has fewer than 2^32 threads, and a grid's second dimension than 2^16)
        const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, (1 << 22) / (row_tiles * shape.split)));
        for (int64_t at = 0; at < y; at += most)
            kernel<<<dim3(row_tiles, (unsigned)std::min(most, y - at), shape.split), 64 * waves, 0, s>>>(m, x, deal, (Out *)x.out, (int)at);
    };
#define BF_GO(GPB, TB, R, W) launch(linear_few_kernel<T, GPB, TB, R, W, DEALT, Out>, TB, R, W)
#define BF_BY_SHAPE(GPB)                                                        \
    if constexpr (DEALT) {                                                      \
        if (shape.waves == 4) BF_GO(GPB, 1, 4, 4);                              \
        else BF_GO(GPB, 1, 2, 8);                                               \
    } else if (shape.tb == 1) {                                                 \
        if (shape.r == 4) BF_GO(GPB, 1, 4, 8);                                  \
        else if (shape.r == 2) BF_GO(GPB, 1, 2, 8);                             \
        else BF_GO(GPB, 1, 1, 8);                                               \
    } else if (shape.tb == 2) {                                                 \
        BF_GO(GPB, 2, few_most_rows<T>, 8);                                     \
    } else if constexpr (sizeof(T) == 2) {                                      \
        if (shape.tb == 3) BF_GO(GPB, 3, 4, 8);                                 \
        else BF_GO(GPB, 4, 4, 8);                                               \
    }
    if (group == 128) { BF_BY_SHAPE(1) }
    else if (group == 64) { BF_BY_SHAPE(2) }
    else { BF_BY_SHAPE(4) }
#undef BF_GO
#undef BF_BY_SHAPE
}

template <typename T>
void by_rows(const Matrices &m, int group, const XRows &x, const Deal *deal, int tiles, bool to_float, const FewShape &shape, hipStream_t s) {
    if (deal) {
        if (to_float) go<T, float, true>(m, group, x, *deal, tiles, shape, s);
        else go<T, T, true>(m, group, x, *deal, tiles, shape, s);
    } else {
        if (to_float) go<T, float, false>(m, group, x, Deal{}, 0, shape, s);
        else go<T, T, false>(m, group, x, Deal{}, 0, shape, s);
    }
}

}  // namespace

hipError_t launch_linear_few(const Matrices &m, int group, const XRows &x, const Deal *deal, int most_tiles, int dtype, bool to_float, const FewShape &shape,
                             hipStream_t s) {
    if (dtype == BIFEAT_F32) by_rows<float>(m, group, x, deal, most_tiles, to_float, shape, s);
    else if (dtype == BIFEAT_F16) by_rows<Half16>(m, group, x, deal, most_tiles, to_float, shape, s);
    else by_rows<Brain16>(m, group, x, deal, most_tiles, to_float, shape, s);
    return hipGetLastError();
}

}  // namespace bf
