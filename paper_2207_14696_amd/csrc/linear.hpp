// Products with matrices in 4 bits: what their translation units share.
//
// With codes q, scale s and minimum m of each group g of a row's columns
//   y = sum_g  s_g sum_{k in g} x_k q_k + m_g sum_{k in g} x_k
//     = sum_g  s_g sum_{k in g} x_k (16 + q_k) + (m_g - 16 s_g) sum_{k in g} x_k.
// 16 + q is a 16-bit float whose highest mantissa bits are q: two codes become two operands of a matrix product by a shift and one
// bitwise instruction, exactly.  With rows of 32 bits the codes are taken as they are (twice the instructions, beside three products): the 16 would
// bring sums three times as large, and cost them 1.5 bits; a 16-bit result has 13 and more to spare.  The products of a group are summed in fp32 by the matrix cores and
// scaled into the result; what sums of x add comes beside them, group by group or a few groups at a time, so that nothing larger than that ever stands in the
// result: of few rows a product with ones has the sum of x (two fused multiply-adds a group), of many a kernel of its own, and another product brings it in.  Neither a
// weight nor a partial sum is ever rounded to 16 bits.
#pragma once

#include "cache.hpp"

namespace bf {

struct Matrices {
    const uint8_t *packed;
    int64_t bytes;  // of one
    int N, K;
    int rows, blocks;  // of 16, and of 128 columns
    int experts;
    __host__ __device__ int64_t code_bytes() const { return (int64_t)rows * blocks * 1024; }
};

typedef float Sum4 __attribute__((ext_vector_type(4)));

// ---- operands of the matrix products.  Pieces: how many of them are a row's value together
template <typename T> struct Operand;
template <> struct Operand<Half16> {
    typedef _Float16 Eight __attribute__((ext_vector_type(8)));
    static constexpr int kPieces = 1;
    static constexpr float kMore = 16.f;  // of a code's operand than the code
    static constexpr uint32_t kMask = 0x03c003c0u, kSixteen = 0x4c004c00u, kOnes = 0x3c003c00u;
    static constexpr int kShift[4] = {6, 2, -2, -6};
    static __device__ Sum4 product(Eight a, Eight b, Sum4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<Brain16> {
    typedef __bf16 Eight __attribute__((ext_vector_type(8)));
    static constexpr int kPieces = 1;
    static constexpr float kMore = 16.f;
    static constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u, kOnes = 0x3f803f80u;
    static constexpr int kShift[4] = {3, -1, -5, -9};
    static __device__ Sum4 product(Eight a, Eight b, Sum4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
// a 32-bit number is three bfloat16 together: 8 bits of it each
template <> struct Operand<float> : Operand<Brain16> {
    static constexpr int kPieces = 3;
    static constexpr float kMore = 0.f;
};

// The eight codes of a word, each with kMore.
template <typename T>
__device__ inline typename Operand<T>::Eight code_operands(uint32_t w) {
    typedef Operand<T> O;
    uint32_t __attribute__((ext_vector_type(4))) r;
    // (in registers, so that one instruction does both; as constants they would be two)
    uint32_t mask = O::kMask, sixteen = O::kSixteen;
    asm("" : "+v"(mask));
    asm("" : "+s"(sixteen));
    if constexpr (O::kMore == 0.f) {
        // (a code is a 32-bit float of which bfloat16 is the upper half)
        const uint32_t even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t from = j % 2 ? odd : even;  // nibble j, and the one 16 bits further
            const float low = (float)(from >> 8 * (j / 2) & 0xffu), high = (float)(from >> (16 + 8 * (j / 2)) & 0xffu);
            r[j] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, high), __builtin_bit_cast(uint32_t, low), 0x07060302u);
        }
        return __builtin_bit_cast(typename O::Eight, r);
    }
#pragma unroll
    for (int j = 0; j < 4; j++) r[j] = ((O::kShift[j] > 0 ? w << (O::kShift[j] & 31) : w >> (-O::kShift[j] & 31)) & mask) | sixteen;
    return __builtin_bit_cast(typename O::Eight, r);
}
template <typename T>
__device__ inline typename Operand<T>::Eight ones() {
    const uint32_t __attribute__((ext_vector_type(4))) r = {Operand<T>::kOnes, Operand<T>::kOnes, Operand<T>::kOnes, Operand<T>::kOnes};
    return __builtin_bit_cast(typename Operand<T>::Eight, r);
}

// Columns: eight of a row of x as they lie in memory (cache.hpp).
// From column `at` of a row of K >= 8, those past the end as zeros: the row's last eight, moved down.
template <typename T>
__device__ inline Columns<T> load_last_columns(const T *row, int at, int K) {
    const int from = at < K - 8 ? at : K - 8, past = at < K ? at - from : 8;
    Columns<T> c = load_columns(row + from);
    constexpr int kWords = 2 * sizeof(T), kPerWord = 4 / sizeof(T);
#pragma unroll
    for (int by = kWords; by >= 1; by /= 2)
#pragma unroll
        for (int i = 0; i < kWords; i++) c.w[i] = past & (by * kPerWord) ? (i + by < kWords ? c.w[i + by < kWords ? i + by : 0] : 0u) : c.w[i];
    if constexpr (kPerWord == 2)
#pragma unroll
        for (int i = 0; i < kWords; i++) c.w[i] = past & 1 ? c.w[i] >> 16 | (i + 1 < kWords ? c.w[i + 1 < kWords ? i + 1 : 0] << 16 : 0u) : c.w[i];
    return c;
}
// ... and as operands
template <typename T>
__device__ inline void to_operands(const Columns<T> &c, typename Operand<T>::Eight (&x)[Operand<T>::kPieces]) {
    if constexpr (Operand<T>::kPieces == 1) {
        x[0] = __builtin_bit_cast(typename Operand<T>::Eight, c);
    } else {
        uint32_t __attribute__((ext_vector_type(4))) r[3];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            // (what is left after the highest 8 bits, and after the next 8, is exact in 32 bits)
            uint32_t piece[3][2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float left = __builtin_bit_cast(float, c.w[2 * j + h]);
#pragma unroll
                for (int p = 0; p < 3; p++) {
                    piece[p][h] = __builtin_bit_cast(uint32_t, left) & 0xffff0000u;
                    left -= __builtin_bit_cast(float, piece[p][h]);
                }
            }
#pragma unroll
            for (int p = 0; p < 3; p++) r[p][j] = piece[p][0] >> 16 | piece[p][1];
        }
#pragma unroll
        for (int p = 0; p < 3; p++) x[p] = __builtin_bit_cast(typename Operand<T>::Eight, r[p]);
    }
}

// ---- the rows of a call
struct XRows {
    const void *x;
    int64_t token_stride, choice_stride;
    int choices;  // rows of a token (1 without experts)
    int64_t count;
    void *out;
    // of many rows, the sums of each group's columns: [sum_rows][groups of all blocks][4] bfloat16, a row of x as often as it lies in memory
    const uint2 *sums;
    int64_t sum_rows;
};

// Where rows are dealt to experts, a tile is up to 16 or kManyRows pairs of a token and one of its choices that name one expert; it has as many places in `order`,
// of which the first `count` are filled.
struct Tile {
    int expert, count;  // expert -1: pairs that name none
};
struct Deal {
    const int *tiles_count;
    const Tile *tiles;
    const int *order;
};

hipError_t launch_linear_pack(const Matrices &m, int group, const void *weight, int dtype, uint8_t *packed, hipStream_t s);
hipError_t launch_linear_unpack(const Matrices &m, int group, float *weight, hipStream_t s);
// How few rows are taken: 16 tb of them and 16 r of the matrix a workgroup, columns in `split` parts (without a deal).
struct FewShape {
    int tb, r, split, waves;
};
template <typename T> constexpr int few_most_rows = sizeof(T) == 4 ? 2 : 4;  // r of tb >= 2
// deal null: one matrix, rows as they are.  to_float: out is fp32 whatever the rows' type; of several parts one after another.
hipError_t launch_linear_few(const Matrices &m, int group, const XRows &x, const Deal *deal, int most_tiles, int dtype, bool to_float, const FewShape &shape,
                             hipStream_t s);
// ... of K >= 8 columns, tiles of kManyRows
constexpr int kManyRows = 128;
hipError_t launch_linear_sums(const Matrices &m, int group, const XRows &x, int dtype, hipStream_t s);
hipError_t launch_linear_many(const Matrices &m, int group, const XRows &x, const Deal *deal, int most_tiles, int dtype, bool to_float, int split, hipStream_t s);
// out = the parts' sum, `count` numbers each
hipError_t launch_linear_add(const float *parts, int split, int64_t count, int dtype, void *out, hipStream_t s);
// Workgroups that deal pairs: several from 4096 on (one then takes longer than a launch more), 2048 or more each, 64 at most.
inline int deal_parts(int64_t pairs) { return pairs < 4096 ? 1 : pairs < 64 * 2048 ? (int)(pairs / 2048) : 64; }
// counts: deal_parts x (experts + 1)
hipError_t launch_linear_deal(const int *ids, int pairs, int experts, int tile, int *counts, int *tiles_count, Tile *tiles, int *order, hipStream_t s);
hipError_t launch_linear_join(const float *products, const int *ids, const float *weights, int64_t tokens, int choices, int experts, int N, int dtype, void *out,
                              hipStream_t s);

}  // namespace bf
