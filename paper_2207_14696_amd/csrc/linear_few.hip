// Products of few rows with matrices in 4 bits.
#include <algorithm>

#include "linear.hpp"

namespace bf {
namespace {

constexpr int kWaves = 8;

// A workgroup takes R times 16 rows of the matrix and up to 16 TB rows of x; its waves take blocks of 128 columns in turn and add up what they have
// in LDS at the end.  A lane's 16 bytes of a block are 32 codes of one row of the matrix, four operands as they are.
template <typename T, int GPB, int TB, int R, bool DEALT, typename Out>
__global__ __launch_bounds__(64 * kWaves) void linear_few_kernel(Matrices m, XRows x, Deal deal, Out *out, int tile0) {
    typedef Operand<T> O;
    constexpr int P = O::kPieces;
    __shared__ Sum4 part[kWaves][R * TB][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 16, quarter = lane / 16;
    const int row0 = blockIdx.x * R;
    const int x_tile = tile0 + blockIdx.y;
    int64_t first = (int64_t)x_tile * 16 * TB;
    int count;
    const uint8_t *packed = m.packed;
    if constexpr (DEALT) {
        if (x_tile >= *deal.tiles_count) return;
        const Tile t = deal.tiles[x_tile];
        first = t.first;
        count = t.count;
        if (t.expert < 0) {
            for (int i = threadIdx.x; i < count * 16 * R; i += 64 * kWaves) {
                const int n = 16 * row0 + i % (16 * R);
                if (n < m.N) out[(int64_t)deal.order[first + i / (16 * R)] * m.N + n] = from_float<Out>(0.f);
            }
            return;
        }
        packed += t.expert * m.bytes;
    } else {
        count = x.count - first < 16 * TB ? (int)(x.count - first) : 16 * TB;
    }
    const T *xr[TB];
    int64_t to[TB];
#pragma unroll
    for (int t = 0; t < TB; t++) {
        const int at = 16 * t + col < count ? 16 * t + col : count - 1;  // (what a row past the last gives is not stored)
        int64_t row = first + at;
        if constexpr (DEALT) row = deal.order[row];
        to[t] = row;
        const int64_t token = DEALT ? (int64_t)((uint32_t)row / (uint32_t)x.choices) : row;
        xr[t] = static_cast<const T *>(x.x) + token * x.token_stride + (DEALT ? (row - token * x.choices) * x.choice_stride : 0);
    }
    const uint32_t *levels = reinterpret_cast<const uint32_t *>(packed + m.code_bytes());
    Sum4 total[R][TB];
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int t = 0; t < TB; t++) total[r][t] = 0.f;
    for (int k = wave; k < m.blocks; k += kWaves) {
        uint4 codes[R], level[R][GPB];
#pragma unroll
        for (int r = 0; r < R; r++) {
            const int row = row0 + r < m.rows ? row0 + r : m.rows - 1;
            codes[r] = reinterpret_cast<const uint4 *>(packed)[((int64_t)row * m.blocks + k) * 64 + lane];
#pragma unroll
            for (int g = 0; g < GPB; g++)
                level[r][g] = *reinterpret_cast<const uint4 *>(levels + (((int64_t)row * m.blocks + k) * GPB + g) * 16 + 4 * quarter);
        }
        Columns<T> columns[4][TB];
        const auto load = [&](auto of) {
#pragma unroll
            for (int w = 0; w < 4; w++)
#pragma unroll
                for (int t = 0; t < TB; t++) columns[w][t] = of(xr[t], 128 * k + 32 * w + 8 * quarter);
        };
        if (128 * (k + 1) <= m.K) load([&](const T *row, int at) { return load_columns(row + at); });
        else if (m.K >= 8) load([&](const T *row, int at) { return load_last_columns(row, at, m.K); });
        else load([&](const T *row, int at) { return at == 0 ? load_short_columns(row, m.K) : no_columns<T>(); });
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
                typename O::Eight a[R];
#pragma unroll
                for (int r = 0; r < R; r++) a[r] = code_operands<T>(w == 0 ? codes[r].x : w == 1 ? codes[r].y : w == 2 ? codes[r].z : codes[r].w);
#pragma unroll
                for (int t = 0; t < TB; t++) {
                    typename O::Eight b[P];
                    to_operands<T>(columns[w][t], b);
#pragma unroll
                    for (int p = 0; p < P; p++) {
                        of_x[t] = O::product(ones<T>(), b[p], of_x[t]);
#pragma unroll
                        for (int r = 0; r < R; r++) sum[r][t] = O::product(a[r], b[p], sum[r][t]);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t word = i == 0 ? level[r][g].x : i == 1 ? level[r][g].y : i == 2 ? level[r][g].z : level[r][g].w;
                    const float scale = __builtin_bit_cast(float, word << 16), low = __builtin_bit_cast(float, word & 0xffff0000u);
                    const float rest = fmaf(-O::kMore, scale, low);
#pragma unroll
                    for (int t = 0; t < TB; t++) total[r][t][i] = fmaf(scale, sum[r][t][i], fmaf(rest, of_x[t][i], total[r][t][i]));
                }
        }
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
        const int r = i / TB, t = i - r * TB, n = 16 * (row0 + r) + 4 * quarter;
        int64_t row = to[0];
#pragma unroll
        for (int j = 1; j < TB; j++) row = t == j ? to[j] : row;
        if (16 * t + col >= count) continue;
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (n + j < m.N) out[row * m.N + n + j] = from_float<Out>(y[j]);
    }
}

template <typename T, typename Out, bool DEALT>
void go(const Matrices &m, int group, const XRows &x, const Deal &deal, int64_t tiles, hipStream_t s) {
    const auto launch = [&](auto kernel, int r, int64_t y) {
        const int row_tiles = (m.rows + r - 1) / r;
        // (a launch has fewer than 2^32 threads, and a grid's second dimension than 2^16)
        const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, (1 << 22) / row_tiles));
        for (int64_t at = 0; at < y; at += most)
            kernel<<<dim3(row_tiles, (unsigned)std::min(most, y - at)), 64 * kWaves, 0, s>>>(m, x, deal, (Out *)x.out, (int)at);
    };
    const bool wide = !DEALT && x.count > 16;
    const int64_t y = DEALT ? tiles : wide ? (x.count + 63) / 64 : (x.count + 15) / 16;
#define BF_GO(GPB)                                                                       \
    if constexpr (!DEALT) {                                                              \
        if (wide) return launch(linear_few_kernel<T, GPB, 4, 1, DEALT, Out>, 1, y);      \
    }                                                                                    \
    launch(linear_few_kernel<T, GPB, 1, 1, DEALT, Out>, 1, y)
    if (group == 128) { BF_GO(1); }
    else if (group == 64) { BF_GO(2); }
    else { BF_GO(4); }
#undef BF_GO
}

template <typename T>
void by_rows(const Matrices &m, int group, const XRows &x, const Deal *deal, int tiles, bool to_float, hipStream_t s) {
    if (!deal) go<T, T, false>(m, group, x, Deal{}, 0, s);
    else if (to_float) go<T, float, true>(m, group, x, *deal, tiles, s);
    else go<T, T, true>(m, group, x, *deal, tiles, s);
}

}  // namespace

hipError_t launch_linear_few(const Matrices &m, int group, const XRows &x, const Deal *deal, int most_tiles, int dtype, bool to_float, hipStream_t s) {
    if (dtype == BIFEAT_F32) by_rows<float>(m, group, x, deal, most_tiles, to_float, s);
    else if (dtype == BIFEAT_F16) by_rows<Half16>(m, group, x, deal, most_tiles, to_float, s);
    else by_rows<Brain16>(m, group, x, deal, most_tiles, to_float, s);
    return hipGetLastError();
}

}  // namespace bf
