// Matrices quantised to 4 bits, and back.
#include "linear.hpp"

namespace bf {
namespace {

// A 32-bit number rounded down, or up, to bfloat16's values.
__device__ inline float brain_below(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x), cut = b & 0xffff0000u;
    return __builtin_bit_cast(float, cut != b && x < 0.f ? cut + 0x10000u : cut);
}
__device__ inline float brain_above(float x) { return -brain_below(-x); }

// A wave packs a block of 16 rows by 128 columns: a lane has the row and columns of its four words, the lanes 16, 32 and 48 further the rest of
// their groups.  Done once a matrix.
template <typename T, int GPB>
__global__ __launch_bounds__(kThreads) void linear_pack_kernel(Matrices m, const T *weight, uint8_t *packed) {
    const int64_t block = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const int lane = threadIdx.x % 64;
    if (block >= (int64_t)m.rows * m.blocks) return;
    const int rows = (int)(block / m.blocks), k = (int)(block - (int64_t)rows * m.blocks), n = 16 * rows + lane % 16;
    weight += (int64_t)blockIdx.y * m.N * m.K + (int64_t)n * m.K;
    packed += blockIdx.y * m.bytes;
    float x[4][8];
    int left[4];
    float mn[GPB], mx[GPB];
    bool bad[GPB];
#pragma unroll
    for (int g = 0; g < GPB; g++) mn[g] = INFINITY, mx[g] = -INFINITY, bad[g] = false;
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const int at = 128 * k + 32 * w + 8 * (lane / 16), g = w * GPB / 4;
        left[w] = n < m.N ? m.K - at : 0;
        load8_any(weight + (left[w] > 0 ? at : 0), left[w], x[w]);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < left[w]) {
                bad[g] |= !(fabsf(x[w][i]) <= 3.402823466e38f);
                mn[g] = fminf(mn[g], x[w][i]);
                mx[g] = fmaxf(mx[g], x[w][i]);
            }
    }
    uint32_t level[GPB];
    float scale[GPB];
#pragma unroll
    for (int g = 0; g < GPB; g++) {
#pragma unroll
        for (int by = 16; by < 64; by *= 2) {
            mn[g] = fminf(mn[g], __shfl_xor(mn[g], by));
            mx[g] = fmaxf(mx[g], __shfl_xor(mx[g], by));
            bad[g] |= __shfl_xor((int)bad[g], by) != 0;
        }
        if (mn[g] > mx[g] && !bad[g]) mn[g] = mx[g] = 0.f;  // no column
        mn[g] = brain_below(mn[g]);
        scale[g] = brain_above((mx[g] - mn[g]) / 15.f);
        if (bad[g] || !(fabsf(mn[g]) <= 3.402823466e38f) || !(scale[g] <= 3.402823466e38f)) mn[g] = scale[g] = NAN;
        level[g] = __builtin_bit_cast(uint32_t, scale[g]) >> 16 | (__builtin_bit_cast(uint32_t, mn[g]) & 0xffff0000u);
    }
    uint32_t word[4];
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const int g = w * GPB / 4;
        word[w] = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float q = scale[g] > 0.f && i < left[w] ? fminf(fmaxf(rintf((x[w][i] - mn[g]) / scale[g]), 0.f), 15.f) : 0.f;
            word[w] |= (uint32_t)q << 4 * (i / 2 + 4 * (i % 2));
        }
    }
    reinterpret_cast<uint4 *>(packed)[block * 64 + lane] = make_uint4(word[0], word[1], word[2], word[3]);
    if (lane < 16)
#pragma unroll
        for (int g = 0; g < GPB; g++) reinterpret_cast<uint32_t *>(packed + m.code_bytes())[(block * GPB + g) * 16 + lane] = level[g];
}

template <int GPB>
__global__ __launch_bounds__(kThreads) void linear_unpack_kernel(Matrices m, float *weight) {
    const int64_t block = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const int lane = threadIdx.x % 64;
    if (block >= (int64_t)m.rows * m.blocks) return;
    const int rows = (int)(block / m.blocks), k = (int)(block - (int64_t)rows * m.blocks), n = 16 * rows + lane % 16;
    if (n >= m.N) return;
    const uint8_t *packed = m.packed + blockIdx.y * m.bytes;
    weight += (int64_t)blockIdx.y * m.N * m.K + (int64_t)n * m.K;
    const uint4 codes = reinterpret_cast<const uint4 *>(packed)[block * 64 + lane];
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const uint32_t word = w == 0 ? codes.x : w == 1 ? codes.y : w == 2 ? codes.z : codes.w;
        const uint32_t level = reinterpret_cast<const uint32_t *>(packed + m.code_bytes())[(block * GPB + w * GPB / 4) * 16 + lane % 16];
        const float scale = __builtin_bit_cast(float, level << 16), low = __builtin_bit_cast(float, level & 0xffff0000u);
        const int at = 128 * k + 32 * w + 8 * (lane / 16);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = fmaf((float)(word >> 4 * (i / 2 + 4 * (i % 2)) & 15u), scale, low);
        if (at < m.K) store_any<8, false>(weight + at, m.K - at, x);
    }
}

dim3 blocks_of(const Matrices &m) { return dim3((unsigned)(((int64_t)m.rows * m.blocks + kThreads / 64 - 1) / (kThreads / 64)), m.experts); }

template <typename T>
void pack(const Matrices &m, int group, const void *weight, uint8_t *packed, hipStream_t s) {
    const auto *w = static_cast<const T *>(weight);
    if (group == 128) linear_pack_kernel<T, 1><<<blocks_of(m), kThreads, 0, s>>>(m, w, packed);
    else if (group == 64) linear_pack_kernel<T, 2><<<blocks_of(m), kThreads, 0, s>>>(m, w, packed);
    else linear_pack_kernel<T, 4><<<blocks_of(m), kThreads, 0, s>>>(m, w, packed);
}

}  // namespace

hipError_t launch_linear_pack(const Matrices &m, int group, const void *weight, int dtype, uint8_t *packed, hipStream_t s) {
    if (dtype == BIFEAT_F32) pack<float>(m, group, weight, packed, s);
    else if (dtype == BIFEAT_F16) pack<Half16>(m, group, weight, packed, s);
    else pack<Brain16>(m, group, weight, packed, s);
    return hipGetLastError();
}

hipError_t launch_linear_unpack(const Matrices &m, int group, float *weight, hipStream_t s) {
    if (group == 128) linear_unpack_kernel<1><<<blocks_of(m), kThreads, 0, s>>>(m, weight);
    else if (group == 64) linear_unpack_kernel<2><<<blocks_of(m), kThreads, 0, s>>>(m, weight);
    else linear_unpack_kernel<4><<<blocks_of(m), kThreads, 0, s>>>(m, weight);
    return hipGetLastError();
}

}  // namespace bf
