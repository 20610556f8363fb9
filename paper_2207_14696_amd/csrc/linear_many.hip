// Products of many rows with matrices in 4 bits.
#include <algorithm>
#include <type_traits>

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

typedef Operand<Brain16>::Eight Brains;

// The sums of each group's columns of the rows of x, each as three bfloat16 that are it together and a zero: sums[row][group][4], groups past the last as zeros.
// A wave takes kRowsOf rows, a lane eight columns; four loads of 512 columns are on their way at a time, of one long row or of four short ones, and 64 groups at
// a time are written side by side.  2048 rows of 4096 columns 5.0 us (a lane each writing what it has 10), 32 768 of 768 10 (20).
template <typename T, int GPB, int kRowsOf>
__global__ __launch_bounds__(kThreads) void linear_sums_kernel(XRows x, int64_t row0, int64_t rows, int K, int groups, uint2 *sums) {
    constexpr int kLanes = 16 / GPB, kChunks = 4 / kRowsOf;  // lanes of a group, loads of a row
    constexpr int kPerChunk = 64 / kLanes;                    // groups
    __shared__ float all[kThreads / 64][kRowsOf][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t r0 = row0 + ((int64_t)blockIdx.x * (kThreads / 64) + wave) * kRowsOf;
    if (r0 >= rows) return;
    const T *row[kRowsOf];
#pragma unroll
    for (int i = 0; i < kRowsOf; i++) {
        const int64_t r = r0 + i < rows ? r0 + i : rows - 1, token = x.choice_stride ? r / x.choices : r;
        row[i] = static_cast<const T *>(x.x) + token * x.token_stride + (x.choice_stride ? (r - token * x.choices) * x.choice_stride : 0);
    }
    for (int g0 = 0; g0 < groups; g0 += 64) {
        const int begin = g0 * 8 * kLanes, end = begin + 512 * kLanes < K ? begin + 512 * kLanes : K;
#pragma unroll
        for (int i = 0; i < kRowsOf; i++) all[wave][i][lane] = 0.f;
        __builtin_amdgcn_wave_barrier();
        for (int from = begin; from < end; from += 512 * kChunks) {
            Columns<T> c[kRowsOf][kChunks];
            const auto bring = [&](auto of) {
#pragma unroll
                for (int i = 0; i < kRowsOf; i++)
#pragma unroll
                    for (int j = 0; j < kChunks; j++) c[i][j] = of(row[i], from + 512 * j + 8 * lane);
            };
            if (from + 512 * kChunks <= K) bring([](const T *r, int at) { return load_columns(r + at); });
            else bring([&](const T *r, int at) { return load_last_columns(r, at, K); });
#pragma unroll
            for (int i = 0; i < kRowsOf; i++)
#pragma unroll
                for (int j = 0; j < kChunks; j++) {
                    float y = sum_of(c[i][j]);
                    y += of_neighbour<0xb1>(y);                               // lane ^ 1
                    y += of_neighbour<0x4e>(y);                               // lane ^ 2
                    if constexpr (kLanes >= 8) y += of_neighbour<0x141>(y);   // the other four of eight
                    if constexpr (kLanes >= 16) y += of_neighbour<0x140>(y);  // the other eight of sixteen
                    const int g = (from - begin) / (8 * kLanes) + j * kPerChunk + lane / kLanes;
                    if (lane % kLanes == 0 && g < 64) all[wave][i][g] = y;
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
#pragma unroll
        for (int i = 0; i < kRowsOf; i++) {
            float y = all[wave][i][lane];
            uint32_t piece[3];
#pragma unroll
            for (int p = 0; p < 3; p++) {
                piece[p] = __builtin_bit_cast(uint32_t, y) & 0xffff0000u;
                y -= __builtin_bit_cast(float, piece[p]);
            }
            if (g0 + lane < groups && r0 + i < rows) sums[(r0 + i) * groups + g0 + lane] = make_uint2(piece[0] >> 16 | piece[1], piece[2] >> 16);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Rows have 8 columns at least.  A workgroup of four waves takes 128 rows of the matrix and 128 of x, a wave 32 of the matrix's and all of x's (64 of each would
// unpack each code twice).  Codes come from memory as the operands that they are; x goes through LDS, by steps of kStep columns, the next but one and the
// one after it on their way while this one's products run.
// What (m_g - 16 s_g) sum x adds is a product too: minimum and scale are bfloat16, the sums three of them (the kernel above), so that one product of 16
// "columns" adds two groups', exactly: of a block of 64 or 128 columns, where a group is 128 of every other block and the one before it (a product a block 305 us at
// 8192 rows, 288 so).  All groups' minima at first would take a product for 16 groups (2048 rows 78 us for 80, in groups of 32 105 for 97), but the result would then
// stand at the size of all minima together, and the 16's, until the sums take them back: hundreds of times its own where the columns of x have a mean.  (x of
// mean and deviation 1 in 32 bits by 8192 columns in groups of 32: an error of 3.3e-5 then, 2.7e-6 now, by few rows' kernel 8.8e-7; by 4096 in groups of 128 2.5e-6
// and 3.4e-6.)
constexpr int kRows = kManyRows;
template <typename T> constexpr int kStep = sizeof(T) == 4 ? 32 : 64;

template <typename X>
__device__ inline X of_bytes(const X *p, uint32_t further) {
    return *reinterpret_cast<const X *>(reinterpret_cast<const uint8_t *>(p) + further);
}

template <typename T, int GPB, bool DEALT, typename Out>
__global__ __launch_bounds__(256, 2) void linear_many_kernel(Matrices m, XRows x, Deal deal, Out *out, int row_tiles, int tile0, int tiles_end) {
    typedef Operand<T> O;
    typedef typename O::Eight Operands;
    constexpr int P = O::kPieces, S = kStep<T>, kChunks = S / 8;
    constexpr int kStride = kRows + 1;  // (of a chunk in 16 bytes: the lanes that write a row's chunks meet no two in a bank)
    __shared__ uint4 tile[2][P][kChunks * kStride];
    constexpr int kPairs = GPB == 4 ? 2 : 1;        // of groups that a block has
    constexpr bool kTwo = GPB == 1 && P == 1;        // where it is one group, two blocks are a pair (of 32-bit rows, for want of registers, each by itself)
    __shared__ uint4 pair_sums[2][kPairs][kRows];  // the sums of x of two groups
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 32, half = lane / 32;
    // Workgroups go to the eight XCDs in turn.  tiles_end > 0: each XCD takes whole tiles of x, whose products with all rows of the matrix find them in its L2
    const int die = blockIdx.x % 8, of_die = blockIdx.x / 8;
    const int n_tile = tiles_end ? of_die % row_tiles : blockIdx.x % row_tiles;
    const int x_tile = tile0 + (tiles_end ? of_die / row_tiles * 8 + die : blockIdx.x / row_tiles);
    if (tiles_end && x_tile >= tiles_end) return;
    const int64_t first = (int64_t)x_tile * kRows;
    int count;
    const uint8_t *packed = m.packed;
    __shared__ int named[DEALT ? kRows : 1];  // the pairs of the tile
    if constexpr (DEALT) {
        // (all of it asked for at a time; places that are not filled are the first one's)
        const int tiles = *deal.tiles_count, head = deal.order[first], mine = deal.order[first + threadIdx.x % kRows];
        const Tile t = deal.tiles[x_tile];
        if (x_tile >= tiles) return;
        count = t.count;
        if (t.expert < 0) {
            for (int i = threadIdx.x; i < count * kRows; i += 256) {
                const int n = kRows * n_tile + i % kRows;
                if (n < m.N) out[(int64_t)deal.order[first + i / kRows] * m.N + n] = from_float<Out>(0.f);
            }
            return;
        }
        packed += t.expert * m.bytes;
        if (threadIdx.x < kRows) named[threadIdx.x] = (int)threadIdx.x < count ? mine : head;
        __syncthreads();
    } else {
        count = x.count - first < kRows ? (int)(x.count - first) : kRows;
    }
    const auto row_of = [&](int i) -> int64_t {  // of the tile's rows (past the last one: one that is there)
        if constexpr (DEALT) return named[i];
        return first + (i < count ? i : count - 1);
    };
    // what a thread brings of x: chunk `threadIdx.x % kChunks` of the rows threadIdx.x / kChunks, + 256 / kChunks, ...
    const int chunk = threadIdx.x % kChunks;
    const auto from_of = [&](int thread, int i) {
        const int64_t row = row_of(thread / kChunks + i * (256 / kChunks)), token = DEALT ? (int64_t)((uint32_t)row / (uint32_t)x.choices) : row;
        return static_cast<const T *>(x.x) + token * x.token_stride + (DEALT ? (row - token * x.choices) * x.choice_stride : 0);
    };
    const int begin = (int)((int64_t)m.blocks * blockIdx.y / gridDim.y), end = (int)((int64_t)m.blocks * (blockIdx.y + 1) / gridDim.y);  // of the columns
    if constexpr (!DEALT) out += blockIdx.y * x.count * m.N;
    const int n0 = kRows * n_tile + 32 * wave;  // the wave's rows of the matrix
    const uint4 *codes = reinterpret_cast<const uint4 *>(packed);
    const uint32_t *all_levels = reinterpret_cast<const uint32_t *>(packed + m.code_bytes());
    const int groups = m.blocks * GPB;
    const auto row16 = [&](int r) { return r < m.rows ? r : m.rows - 1; };
    // (the wave's part of an address, and the lane's in 32 bits: fewer registers)
    const int rows0 = row16(n0 / 16);
    const uint32_t lane_rows = row16(n0 / 16 + col / 16) - rows0;
    // The products with 32 J rows of x.
    const auto run = [&](auto wide) {
        constexpr int J = decltype(wide)::value, L = (32 * J * kChunks + 255) / 256;  // (loads that reach them)
        Sum16 total[J], sum[J];
#pragma unroll
        for (int j = 0; j < J; j++) total[j] = 0.f;

        const T *from[L];
        {
            int thread = threadIdx.x;  // (worked out here, and again for the last columns: they would be kept from the other widths' beginnings, or beside what the loop counts up)
            asm("" : "+v"(thread));
#pragma unroll
            for (int i = 0; i < L; i++) from[i] = from_of(thread, i);
        }
        Columns<T> coming[2][L];  // of the next steps, by turns
        const auto bring = [&](int step, Columns<T> (&c)[L]) {
#pragma unroll
            for (int i = 0; i < L; i++) c[i] = load_columns(from[i] + S * step + 8 * chunk);
        };
        const auto put = [&](int part, const Columns<T> (&c)[L]) {  // what has come, of a block's part
#pragma unroll
            for (int i = 0; i < L; i++) {
                const int at = threadIdx.x / kChunks + i * (256 / kChunks);
                Operands b[P];
                to_operands<T>(c[i], b);
#pragma unroll
                for (int p = 0; p < P; p++) tile[part & 1][p][chunk * kStride + at] = __builtin_bit_cast(uint4, b[p]);
            }
        };
        const uint32_t *my_levels = all_levels + (int64_t)rows0 * groups * 16;
        const uint32_t levels_at = (lane_rows * groups * 16 + col % 16) * 4;
        uint32_t level[GPB], level_now[GPB] = {}, level_before = 0;
        const auto bring_levels = [&](int k) {
#pragma unroll
            for (int g = 0; g < GPB; g++) level[g] = of_bytes(my_levels + (k * GPB + g) * 16, levels_at);
        };
        const uint4 *my_codes = codes + (int64_t)rows0 * m.blocks * 64;
        const uint32_t codes_at = (lane_rows * m.blocks * 64 + col % 16 + 16 * half) * 16;
        uint4 a[2], now[2];
        const auto bring_codes = [&](int k) {
#pragma unroll
            for (int e = 0; e < 2; e++) a[e] = of_bytes(my_codes + (int64_t)k * 64 + 32 * e, codes_at);
        };
        const auto take = [&] {
            level_before = level_now[0];
#pragma unroll
            for (int e = 0; e < 2; e++) now[e] = a[e];
#pragma unroll
            for (int g = 0; g < GPB; g++) level_now[g] = level[g];
        };
        constexpr int kParts = 128 / S;
        // What a pair of groups' minima add, of the block r after the first (where two are a pair the block before it besides, of odd r).
        uint4 of[J];
        const auto read_sums = [&](int r, int pair) {
#pragma unroll
            for (int j = 0; j < J; j++) of[j] = pair_sums[(kTwo ? r / 2 : r) & 1][pair][32 * j + col];
        };
        constexpr int kDeep = P == 1 ? 2 : 1;  // (of three pieces two would not fit the registers)
        const auto add_minima = [&](int r, int pair, bool both) {
            const bool two = kTwo && both;
            uint32_t __attribute__((ext_vector_type(4))) rest;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const uint32_t w = GPB > 1 ? level_now[GPB > 1 ? 2 * pair + i : 0] : i == 0 && two ? level_before : i == 0 || two ? level_now[0] : 0u;
                // the lower half of the lanes has minima, the upper one -kMore scales (the sign, and 4 more in the exponent; a scale of 0 stays it, the largest ones pass
                // what the header allows)
                uint32_t more = 0;
                if constexpr (O::kMore != 0.f) more = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, w << 16) * -O::kMore);
                const uint32_t v = half ? more : w;  // (in its upper 16 bits)
                rest[2 * i] = __builtin_amdgcn_perm(v, v, 0x07060706u);
                rest[2 * i + 1] = v >> 16;
            }
#pragma unroll
            for (int j = 0; j < J; j++) {
                uint4 a = kDeep == 1 ? pair_sums[r & 1][pair][32 * j + col] : of[j];
                if (GPB == 1 && !two) a.z = a.w = 0;
                total[j] = product32<Brain16>(__builtin_bit_cast(Brains, a), __builtin_bit_cast(Brains, rest), total[j]);
                if (kDeep == 1) __builtin_amdgcn_sched_barrier(0);
            }
        };
        const auto multiply = [&](int r, int part, bool minima, bool both) {
            Operands b[kDeep][J][P];
            const auto read = [&](int s16) {
#pragma unroll
                for (int j = 0; j < J; j++)
#pragma unroll
                    for (int p = 0; p < P; p++)
                        b[s16 % kDeep][j][p] = __builtin_bit_cast(Operands, tile[part & 1][p][(2 * s16 + half) * kStride + 32 * j + col]);
            };
            constexpr int kPerPair = kParts / kPairs;
            constexpr bool kAhead = kDeep == 2 && GPB > 1;
            if (kAhead && part % kPerPair == 0) read_sums(r, part / kPerPair);
            if (kDeep == 2) read(0);
            else if (part % kPerPair == 0) {  // (before x takes the registers)
                add_minima(r, part / kPerPair, both);
                __builtin_amdgcn_sched_barrier(0);
            }
            // (a wave's products before the other wave's other work: two waves that keep in step would both wait for the matrix cores, then both for the vector ones;
            // 8192 rows 291 us, 281 so)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int s16 = 0; s16 < S / 16; s16++) {
                const int s = part * (S / 16) + s16;  // of the block's eight
                constexpr int kPer = 8 / GPB;         // 16 columns at a time, of a group
                if (kDeep == 1) read(s16);
                else if (s16 + 1 < S / 16) read(s16 + 1);
                __builtin_amdgcn_sched_barrier(0x11);  // (reads stay ahead of the products)
                const uint4 w = now[s % 2];
                const Operands c = code_operands<T>(s / 2 == 0 ? w.x : s / 2 == 1 ? w.y : s / 2 == 2 ? w.z : w.w);
#pragma unroll
                for (int j = 0; j < J; j++)
#pragma unroll
                    for (int p = 0; p < P; p++) {
                        if (s % kPer == 0 && p == 0) {
                            Sum16 zero;
#pragma unroll
                            for (int e = 0; e < 16; e++) zero[e] = 0.f;
                            sum[j] = product32<T>(b[s16 % kDeep][j][p], c, zero);
                        } else {
                            sum[j] = product32<T>(b[s16 % kDeep][j][p], c, sum[j]);
                        }
                    }
                if (kDeep == 2 && part % kPerPair == 0 && s16 == 0 && minima) {
                    if (!kAhead) read_sums(r, part / kPerPair);
                    add_minima(r, part / kPerPair, both);
                }
                if (s % kPer == kPer - 1) {
                    const int g = s / kPer;
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(0);
                    const float scale = __builtin_bit_cast(float, level_now[g] << 16);
#pragma unroll
                    for (int j = 0; j < J; j++)
#pragma unroll
                        for (int e = 0; e < 16; e++) total[j][e] = fmaf(scale, sum[j][e], total[j][e]);
                    // (here and not where they are used next: the compiler would keep what they are made of until then)
#pragma unroll
                    for (int j = 0; j < J; j++) asm volatile("" : "+v"(total[j]));
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(1);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        };
        // A block's sums of x: a thread brings half of a row's.
        const uint32_t *my_sums = reinterpret_cast<const uint32_t *>(x.sums) + GPB * (threadIdx.x % 2);
        {
            int64_t row = row_of(threadIdx.x / 2);
            if (DEALT && !x.choice_stride) row = (int64_t)((uint32_t)row / (uint32_t)x.choices);
            my_sums += row * groups * 2;
        }
        typedef uint32_t HalfSums __attribute__((ext_vector_type(GPB)));
        HalfSums half_sums;
        const auto bring_sums = [&](int k) { half_sums = *reinterpret_cast<const HalfSums *>(my_sums + (int64_t)k * GPB * 2); };
        const auto put_sums = [&](int r) {
            const int row = threadIdx.x / 2, of = threadIdx.x % 2;
            uint4 *to = &pair_sums[(kTwo ? r / 2 : r) & 1][kPairs == 2 ? of : 0][row];
            *reinterpret_cast<HalfSums *>(reinterpret_cast<uint32_t *>(to) + (kTwo ? 2 * (r & 1) + of : GPB * of % 4)) = half_sums;
        };
        // Whole blocks: no branch leads to a load, so that none is waited for before its use; what is asked for past the last step is the last again.
        const int whole = end < m.K / 128 ? end : m.K / 128;
        if (begin < whole) {
            const int last = whole * kParts - 1;
            bring(begin * kParts, coming[0]);
            bring(begin * kParts + 1, coming[1]);
            bring_levels(begin);
            bring_codes(begin);
            bring_sums(begin);
            put(0, coming[0]);
            put_sums(0);
            bring(begin * kParts + 2 < last ? begin * kParts + 2 : last, coming[0]);
            bring_sums(begin + 1 < whole ? begin + 1 : begin);
            __syncthreads();
            for (int k = begin; k < whole; k++) {
                const int next = k + 1 < whole ? k + 1 : k;
                take();
                bring_codes(next);
                bring_levels(next);
                put_sums(k - begin + 1);
                bring_sums(k + 2 < whole ? k + 2 : whole - 1);
#pragma unroll
                for (int part = 0; part < kParts; part++) {
                    const int ahead = k * kParts + part + 3;
                    put((part + 1) % kParts, coming[(part + 1) & 1]);
                    bring(ahead < last ? ahead : last, coming[(part + 1) & 1]);
                    multiply(k - begin, part, !kTwo || (k - begin) & 1, true);
                    __syncthreads();
                }
            }
        }
        if (kTwo && whole == end && (whole - begin) & 1) {  // (a block without another)
            read_sums(whole - begin - 1, 0);
            add_minima(whole - begin - 1, 0, false);
        }
        if (whole < end) {  // the rows' last columns
            bring_levels(whole);
            bring_codes(whole);
            bring_sums(whole);
            put_sums(whole - begin);
            take();
            int again = threadIdx.x;
            asm("" : "+v"(again));
#pragma unroll
            for (int part = 0; part < kParts; part++) {
#pragma unroll
                for (int i = 0; i < L; i++) coming[0][i] = load_last_columns(from_of(again, i), 128 * whole + S * part + 8 * chunk, m.K);
                put(part, coming[0]);
                __syncthreads();
                multiply(whole - begin, part, true, (whole - begin) & 1);
                __syncthreads();
            }
        }
        const int n = n0 + col;
#pragma unroll
        for (int j = 0; j < J; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const int at = 32 * j + 8 * (e / 4) + 4 * half + e % 4;
                if (at < count && n < m.N) out[row_of(at) * m.N + n] = from_float<Out>(total[j][e]);
            }
    };
    // (The last tile of an expert's is rarely full: 128 of 2048 x 768 with 40 pairs each 89 us by whole tiles, 58 so, with 256 200 and 182; 300 rows of one of
    // 14336 x 4096 63 and 52.)
    if (count <= 32) return run(std::integral_constant<int, 1>{});
    if (count <= 64) return run(std::integral_constant<int, 2>{});
    if (count <= 96) return run(std::integral_constant<int, 3>{});
    run(std::integral_constant<int, 4>{});
}

template <typename T, typename Out, bool DEALT>
void go(const Matrices &m, int group, const XRows &x, const Deal &deal, int tiles, int split, hipStream_t s) {
    const int row_tiles = (m.N + kRows - 1) / kRows;
    const int64_t all = DEALT ? (int64_t)tiles : (x.count + kRows - 1) / kRows;
    // (a launch has fewer than 2^32 threads)
    const int64_t most = std::max<int64_t>(8, (1 << 22) / (row_tiles * split) / 8 * 8);
    for (int64_t at = 0; at < all; at += most) {
        const int64_t here = std::min(most, all - at);
        const bool whole = here % 8 == 0 || here >= 64;
        const dim3 grid((unsigned)(row_tiles * (whole ? (here + 7) / 8 * 8 : here)), split);
        const int end = whole ? (int)(at + here) : 0;
        if (group == 128) linear_many_kernel<T, 1, DEALT, Out><<<grid, 256, 0, s>>>(m, x, deal, (Out *)x.out, row_tiles, (int)at, end);
        else if (group == 64) linear_many_kernel<T, 2, DEALT, Out><<<grid, 256, 0, s>>>(m, x, deal, (Out *)x.out, row_tiles, (int)at, end);
        else linear_many_kernel<T, 4, DEALT, Out><<<grid, 256, 0, s>>>(m, x, deal, (Out *)x.out, row_tiles, (int)at, end);
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

hipError_t launch_linear_sums(const Matrices &m, int group, const XRows &x, int dtype, hipStream_t s) {
    const int64_t rows = x.sum_rows;
    const int of = m.K > 1024 ? 1 : 4;
    const int64_t per = kThreads / 64 * of, most = per << 23;  // (a launch has fewer than 2^32 threads)
    uint2 *sums = const_cast<uint2 *>(x.sums);
#define BF_RUN(T, GPB)                                                                                                          \
    if (of == 1) linear_sums_kernel<T, GPB, 1><<<grid, kThreads, 0, s>>>(x, row0, rows, m.K, m.blocks * GPB, sums);                    \
    else linear_sums_kernel<T, GPB, 4><<<grid, kThreads, 0, s>>>(x, row0, rows, m.K, m.blocks * GPB, sums)
#define BF_GO(T)                                  \
    if (group == 128) { BF_RUN(T, 1); }           \
    else if (group == 64) { BF_RUN(T, 2); }       \
    else { BF_RUN(T, 4); }
    for (int64_t row0 = 0; row0 < rows; row0 += most) {
        const unsigned grid = (unsigned)(((rows - row0 < most ? rows - row0 : most) + per - 1) / per);
        if (dtype == BIFEAT_F32) { BF_GO(float); }
        else if (dtype == BIFEAT_F16) { BF_GO(Half16); }
        else { BF_GO(Brain16); }
    }
#undef BF_GO
#undef BF_RUN
    return hipGetLastError();
}

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
