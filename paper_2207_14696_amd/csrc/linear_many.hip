// Products of many rows with matrices in 4 bits.
#include <algorithm>

#include "linear.hpp"

namespace bf {
namespace {

typedef float Sum16 __attribute__((ext_vector_type(16)));

template <typename T>
__device__ inline Sum16 product32(typename Operand<T>::Eight a, typename Operand<T>::Eight b, Sum16 c) {
    if constexpr (sizeof(T) == 2 && Operand<T>::kOnes == 0x3c003c00u) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Eight columns of x added up.
template <typename T>
__device__ inline float sum_of(const Columns<T> &c) {
    float y = 0.f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; i++) y += __builtin_bit_cast(float, c.w[i]);
    } else if constexpr (Operand<T>::kOnes == 0x3c003c00u) {
        typedef _Float16 Two __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; i++) y = __builtin_amdgcn_fdot2(__builtin_bit_cast(Two, c.w[i]), Two{(_Float16)1, (_Float16)1}, y, false);
    } else {
        typedef __bf16 Two __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; i++) y = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Two, c.w[i]), Two{(__bf16)1.f, (__bf16)1.f}, y, false);
    }
    return y;
}

template <int CTRL>
__device__ inline float of_neighbour(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// Rows have 8 columns at least.  A workgroup of four waves takes 128 rows of the matrix and 128 of x, a wave 64 of each.  Codes come from memory as the operands that they are; x goes through
// LDS, by steps of kStep columns, the next two steps' on their way while this one's products run; each four lanes that bring 32 columns of a row add them up on the
// way.
constexpr int kRows = kManyRows;
template <typename T> constexpr int kStep = sizeof(T) == 4 ? 32 : 64;

template <typename T, int GPB, bool DEALT, typename Out>
__global__ __launch_bounds__(256, 2) void linear_many_kernel(Matrices m, XRows x, Deal deal, Out *out, int row_tiles, int tile0) {
    typedef Operand<T> O;
    typedef typename O::Eight Operands;
    constexpr int P = O::kPieces, S = kStep<T>, kChunks = S / 8, kLoads = kRows * kChunks / 256;
    constexpr int kStride = kRows + 1;  // (of a chunk in 16 bytes: the lanes that write a row's chunks meet no two in a bank)
    __shared__ uint4 tile[2][P][kChunks * kStride];
    __shared__ float sums[2][GPB][kRows];       // [of this block, the next][group]: of x
    __shared__ float levels[2][2][GPB][kRows];  // [of this block, the next][scale, rest]
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 32, half = lane / 32;
    const int n_tile = blockIdx.x % row_tiles, x_tile = tile0 + blockIdx.x / row_tiles;
    int64_t first = (int64_t)x_tile * kRows;
    int count;
    const uint8_t *packed = m.packed;
    if constexpr (DEALT) {
        if (x_tile >= *deal.tiles_count) return;
        const Tile t = deal.tiles[x_tile];
        first = t.first;
        count = t.count;
        if (t.expert < 0) {
            for (int i = threadIdx.x; i < count * kRows; i += 256) {
                const int n = kRows * n_tile + i % kRows;
                if (n < m.N) out[(int64_t)deal.order[first + i / kRows] * m.N + n] = from_float<Out>(0.f);
            }
            return;
        }
        packed += t.expert * m.bytes;
    } else {
        count = x.count - first < kRows ? (int)(x.count - first) : kRows;
    }
    // what a thread brings of x: chunk `threadIdx.x % kChunks` of the rows threadIdx.x / kChunks, + 256 / kChunks, ...
    const int chunk = threadIdx.x % kChunks;
    const T *from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int at = threadIdx.x / kChunks + i * (256 / kChunks);
        int64_t row = first + (at < count ? at : count - 1);
        if constexpr (DEALT) row = deal.order[row];
        const int64_t token = DEALT ? (int64_t)((uint32_t)row / (uint32_t)x.choices) : row;
        from[i] = static_cast<const T *>(x.x) + token * x.token_stride + (DEALT ? (row - token * x.choices) * x.choice_stride : 0);
    }
    const int begin = (int)((int64_t)m.blocks * blockIdx.y / gridDim.y), end = (int)((int64_t)m.blocks * (blockIdx.y + 1) / gridDim.y);  // of the columns
    if constexpr (!DEALT) out += blockIdx.y * x.count * m.N;
    const int n0 = kRows * n_tile + 64 * (wave % 2), t0 = 64 * (wave / 2);  // the wave's part
    const uint4 *codes = reinterpret_cast<const uint4 *>(packed);
    const uint32_t *all_levels = reinterpret_cast<const uint32_t *>(packed + m.code_bytes());
    const int groups = m.blocks * GPB;
    const auto row16 = [&](int r) { return r < m.rows ? r : m.rows - 1; };
    Sum16 total[2][2], sum[2][2];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++) total[i][j] = 0.f;

    Columns<T> coming[2][kLoads];  // of the next step, and of the one after it
    const auto bring = [&](int step, Columns<T> (&c)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) c[i] = load_columns(from[i] + S * step + 8 * chunk);
    };
    constexpr int kGroup = 128 / GPB, kPerGroup = kGroup > S ? kGroup / S : 1;  // steps
    constexpr int kLanes = (kGroup < S ? kGroup : S) / 8;                        // that bring a row's columns of a group
    float so_far[kLoads];
    const auto put = [&](int k, int part, const Columns<T> (&c)[kLoads]) {  // what has come, of part `part` of block k
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int at = threadIdx.x / kChunks + i * (256 / kChunks);
            Operands b[P];
            to_operands<T>(c[i], b);
#pragma unroll
            for (int p = 0; p < P; p++) tile[part & 1][p][chunk * kStride + at] = __builtin_bit_cast(uint4, b[p]);
            float y = sum_of(c[i]);
            if (part % kPerGroup != 0) y += so_far[i];
            so_far[i] = y;
            if (part % kPerGroup == kPerGroup - 1) {
                y += of_neighbour<0xb1>(y);                        // lane ^ 1
                y += of_neighbour<0x4e>(y);                        // lane ^ 2
                if constexpr (kLanes == 8) y += of_neighbour<0x141>(y);  // the other four of eight
                if (chunk % kLanes == 0) sums[k & 1][(S * part + 8 * chunk) / kGroup][at] = y;
            }
        }
    };
    uint32_t level[GPB];
    const auto bring_levels = [&](int k) {  // of block k: a thread has a row, as another one has
        const int n = threadIdx.x % kRows, r = row16(kRows / 16 * n_tile + n / 16);
#pragma unroll
        for (int g = 0; g < GPB; g++) level[g] = all_levels[((int64_t)r * groups + k * GPB + g) * 16 + n % 16];
    };
    const auto put_levels = [&](int buffer) {
        if (threadIdx.x < kRows)
#pragma unroll
            for (int g = 0; g < GPB; g++) {
                const float scale = __builtin_bit_cast(float, level[g] << 16), low = __builtin_bit_cast(float, level[g] & 0xffff0000u);
                levels[buffer][0][g][threadIdx.x] = scale;
                levels[buffer][1][g][threadIdx.x] = fmaf(-O::kMore, scale, low);
            }
    };
    const uint4 *my_codes[2];
#pragma unroll
    for (int i = 0; i < 2; i++) my_codes[i] = codes + (int64_t)row16(n0 / 16 + 2 * i + col / 16) * m.blocks * 64 + col % 16 + 16 * half;
    uint4 a[2][2], now[2][2];
    const auto bring_codes = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int e = 0; e < 2; e++) a[i][e] = my_codes[i][(int64_t)k * 64 + 32 * e];
    };
    const auto take_codes = [&] {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int e = 0; e < 2; e++) now[i][e] = a[i][e];
    };
    const auto multiply = [&](int k, int part) {
#pragma unroll
        for (int s16 = 0; s16 < S / 16; s16++) {
            const int s = part * (S / 16) + s16;  // of the block's eight
            constexpr int kPer = 8 / GPB;         // 16 columns at a time, of a group
            const bool begins = s % kPer == 0;
            Operands b[2][P];
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int p = 0; p < P; p++)
                    b[j][p] = __builtin_bit_cast(Operands, tile[part & 1][p][(2 * s16 + half) * kStride + t0 + 32 * j + col]);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const uint4 w = now[i][s % 2];
                const Operands c = code_operands<T>(s / 2 == 0 ? w.x : s / 2 == 1 ? w.y : s / 2 == 2 ? w.z : w.w);
#pragma unroll
                for (int j = 0; j < 2; j++) {
#pragma unroll
                    for (int p = 0; p < P; p++) {
                        if (begins && p == 0) {
                            Sum16 zero;
#pragma unroll
                            for (int e = 0; e < 16; e++) zero[e] = 0.f;
                            sum[i][j] = product32<T>(b[j][p], c, zero);
                        } else {
                            sum[i][j] = product32<T>(b[j][p], c, sum[i][j]);
                        }
                    }
                }
            }
            if (s % kPer == kPer - 1) {
                const int g = s / kPer;
                __builtin_amdgcn_sched_barrier(0);
                float scale[2], rest[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    scale[i] = levels[k & 1][0][g][64 * (wave % 2) + 32 * i + col];
                    rest[i] = levels[k & 1][1][g][64 * (wave % 2) + 32 * i + col];
                }
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const Sum4 of_x = *reinterpret_cast<const Sum4 *>(&sums[k & 1][g][t0 + 32 * j + 8 * e + 4 * half]);
#pragma unroll
                        for (int i = 0; i < 2; i++)
#pragma unroll
                            for (int c = 0; c < 4; c++)
                                total[i][j][4 * e + c] = fmaf(scale[i], sum[i][j][4 * e + c], fmaf(rest[i], of_x[c], total[i][j][4 * e + c]));
                    }
                // (here and not where they are used next: the compiler would keep what they are made of until then)
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int j = 0; j < 2; j++) asm volatile("" : "+v"(total[i][j]));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // Whole blocks: no branch leads to a load, so that none is waited for before its use; what is asked for past the last step is the last again.
    constexpr int kParts = 128 / S;
    const int whole = end < m.K / 128 ? end : m.K / 128;
    if (begin < whole) {
        const int last = whole * kParts - 1;
        bring(begin * kParts, coming[0]);
        bring(begin * kParts + 1, coming[1]);
        bring_levels(begin);
        bring_codes(begin);
        put(begin, 0, coming[0]);
        put_levels(begin & 1);
        __syncthreads();
        for (int k = begin; k < whole; k++) {
            const int next = k + 1 < whole ? k + 1 : k;
            take_codes();
            bring_codes(next);
            bring_levels(next);
#pragma unroll
            for (int part = 0; part < kParts; part++) {
                const int ahead = k * kParts + part + 2;
                bring(ahead < last ? ahead : last, coming[part & 1]);
                put(part == kParts - 1 ? k + 1 : k, (part + 1) % kParts, coming[(part + 1) & 1]);
                multiply(k, part);
                if (part == kParts - 1) put_levels((k + 1) & 1);
                __syncthreads();
            }
        }
    }
    if (whole < end) {  // the rows' last columns
        bring_levels(whole);
        bring_codes(whole);
        put_levels(whole & 1);
        take_codes();
#pragma unroll
        for (int part = 0; part < kParts; part++) {
#pragma unroll
            for (int i = 0; i < kLoads; i++) coming[0][i] = load_last_columns(from[i], 128 * whole + S * part + 8 * chunk, m.K);
            put(whole, part, coming[0]);
            __syncthreads();
            multiply(whole, part);
            __syncthreads();
        }
    }
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const int at = t0 + 32 * j + 8 * (e / 4) + 4 * half + e % 4;
            if (at >= count) continue;
            int64_t row = first + at;
            if constexpr (DEALT) row = deal.order[row];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int n = n0 + 32 * i + col;
                if (n < m.N) out[row * m.N + n] = from_float<Out>(total[i][j][e]);
            }
        }
}

template <typename T, typename Out, bool DEALT>
void go(const Matrices &m, int group, const XRows &x, const Deal &deal, int tiles, int split, hipStream_t s) {
    const int row_tiles = (m.N + kRows - 1) / kRows;
    const int64_t all = DEALT ? (int64_t)tiles : (x.count + kRows - 1) / kRows;
    // (a launch has fewer than 2^32 threads)
    const int64_t most = std::max<int64_t>(1, (1 << 22) / (row_tiles * split));
    for (int64_t at = 0; at < all; at += most) {
        const dim3 grid((unsigned)(row_tiles * std::min(most, all - at)), split);
        if (group == 128) linear_many_kernel<T, 1, DEALT, Out><<<grid, 256, 0, s>>>(m, x, deal, (Out *)x.out, row_tiles, (int)at);
        else if (group == 64) linear_many_kernel<T, 2, DEALT, Out><<<grid, 256, 0, s>>>(m, x, deal, (Out *)x.out, row_tiles, (int)at);
        else linear_many_kernel<T, 4, DEALT, Out><<<grid, 256, 0, s>>>(m, x, deal, (Out *)x.out, row_tiles, (int)at);
    }
}

template <typename T>
void by_rows(const Matrices &m, int group, const XRows &x, const Deal *deal, int tiles, bool to_float, int split, hipStream_t s) {
    if (deal) {
        if (to_float) go<T, float, true>(m, group, x, *deal, tiles, split, s);
        else go<T, T, true>(m, group, x, *deal, tiles, split, s);
    } else {
        if (to_float) go<T, float, false>(m, group, x, Deal{}, 0, split, s);
        else go<T, T, false>(m, group, x, Deal{}, 0, split, s);
    }
}

// Four numbers a lane, all parts of them on their way at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_add_kernel(const float *parts, int split, int64_t count, T *out) {
    struct __attribute__((packed, aligned(4))) Four {
        float v[4];
    };
    const int64_t at = 4 * ((int64_t)blockIdx.x * kThreads + threadIdx.x);
    if (at >= count) return;
    const int left = count - at < 4 ? (int)(count - at) : 4;
    float y[4] = {};
    for (int p0 = 0; p0 < split; p0 += 8) {
        Four f[8];
#pragma unroll
        for (int p = 0; p < 8; p++) {
            const float *from = parts + (p0 + p < split ? p0 + p : p0) * count + at;
            if (left == 4) f[p] = *reinterpret_cast<const Four *>(from);
            else
#pragma unroll
                for (int c = 0; c < 4; c++) f[p].v[c] = c < left ? from[c] : 0.f;
        }
#pragma unroll
        for (int p = 0; p < 8; p++)
#pragma unroll
            for (int c = 0; c < 4; c++) y[c] += p0 + p < split ? f[p].v[c] : 0.f;
    }
    store_any<4, false>(out + at, left, y);
}

}  // namespace

hipError_t launch_linear_many(const Matrices &m, int group, const XRows &x, const Deal *deal, int most_tiles, int dtype, bool to_float, int split, hipStream_t s) {
    if (dtype == BIFEAT_F32) by_rows<float>(m, group, x, deal, most_tiles, to_float, split, s);
    else if (dtype == BIFEAT_F16) by_rows<Half16>(m, group, x, deal, most_tiles, to_float, split, s);
    else by_rows<Brain16>(m, group, x, deal, most_tiles, to_float, split, s);
    return hipGetLastError();
}

hipError_t launch_linear_add(const float *parts, int split, int64_t count, int dtype, void *out, hipStream_t s) {
    const unsigned grid = (unsigned)((count + 4 * kThreads - 1) / (4 * kThreads));
    if (dtype == BIFEAT_F32) linear_add_kernel<<<grid, kThreads, 0, s>>>(parts, split, count, (float *)out);
    else if (dtype == BIFEAT_F16) linear_add_kernel<<<grid, kThreads, 0, s>>>(parts, split, count, (Half16 *)out);
    else linear_add_kernel<<<grid, kThreads, 0, s>>>(parts, split, count, (Brain16 *)out);
    return hipGetLastError();
}

}  // namespace bf
