// Tokens' choices dealt to the experts that they name, and the experts' products joined.
#include <algorithm>

#include "linear.hpp"

namespace bf {
namespace {

constexpr int kDealThreads = 1024, kMostExperts = 1024;

__device__ inline int expert_of(int e, int experts) { return e >= 0 && e < experts ? e : experts; }

// A thread's pairs of a part of them, and their experts (those that name none: `experts`; past the end: -1), loads ahead of their use.
constexpr int kPairsAhead = 4;
struct Pairs {
    int first, e[kPairsAhead];
};
__device__ inline Pairs pairs_of(const int *ids, int first, int last, int experts) {
    Pairs p;
    p.first = first;
#pragma unroll
    for (int j = 0; j < kPairsAhead; j++) p.e[j] = first + j * kDealThreads < last ? ids[first + j * kDealThreads] : 0;
#pragma unroll
    for (int j = 0; j < kPairsAhead; j++) p.e[j] = first + j * kDealThreads < last ? expert_of(p.e[j], experts) : -1;
    return p;
}
template <typename F>
__device__ inline void each_of(const Pairs &p, F f) {
#pragma unroll
    for (int j = 0; j < kPairsAhead; j++)
        if (p.e[j] >= 0) f(p.first + j * kDealThreads, p.e[j]);
}

// How many pairs of each part name each expert: counts[part][expert].
__global__ __launch_bounds__(kDealThreads) void linear_count_kernel(const int *ids, int pairs, int per_part, int experts, int *counts) {
    __shared__ int count[kMostExperts + 1];
    for (int e = threadIdx.x; e <= experts; e += kDealThreads) count[e] = 0;
    __syncthreads();
    const int first = blockIdx.x * per_part, last = pairs - first < per_part ? pairs : first + per_part;
    for (int i = first + threadIdx.x; i < last; i += kPairsAhead * kDealThreads)
        each_of(pairs_of(ids, i, last, experts), [&](int, int e) { atomicAdd(&count[e], 1); });
    __syncthreads();
    for (int e = threadIdx.x; e <= experts; e += kDealThreads) counts[blockIdx.x * (experts + 1) + e] = count[e];
}

// Pairs of a token and a choice, expert by expert, in tiles of up to `tile` of one expert's, a power of two; a tile has that many places in `order`, so that its
// pairs are found without knowing it.  The order of an expert's pairs is not fixed; their products do
// not depend on it.  Those that name no expert come last, as an expert of their own.  A workgroup places a part of the pairs; one part is counted
// here, of several `counts` has the numbers.  32 768 pairs of 128 experts in one part 30 us, in 16 3 + 4.
__global__ __launch_bounds__(kDealThreads) void linear_deal_kernel(const int *ids, int pairs, int per_part, int experts, int tile, const int *counts,
                                                                   int *tiles_count, Tile *tiles, int *order) {
    __shared__ int count[kMostExperts + 1], first[kMostExperts + 1], tile_at[kMostExperts + 1];  // first: of this part's, among the expert's
    __shared__ int sums[kDealThreads / 64];
    const int begin = blockIdx.x * per_part, end = pairs - begin < per_part ? pairs : begin + per_part;
    const Pairs mine = pairs_of(ids, begin + threadIdx.x, end, experts);  // (of a part of up to 4096 all)
    if (counts) {
        for (int e = threadIdx.x; e <= experts; e += kDealThreads) {
            int all = 0, earlier = 0;  // ... and what the parts before this one have
            for (int p = 0; p < (int)gridDim.x; p++) {
                const int c = counts[p * (experts + 1) + e];
                all += c;
                earlier += p < (int)blockIdx.x ? c : 0;
            }
            count[e] = all;
            first[e] = earlier;
        }
    } else {
        for (int e = threadIdx.x; e <= experts; e += kDealThreads) count[e] = first[e] = 0;
        __syncthreads();
        each_of(mine, [&](int, int e) { atomicAdd(&count[e], 1); });  // (one part is not longer)
    }
    __syncthreads();
    // the tiles before each expert's: a thread an expert, the last those of none besides
    const int c = (int)threadIdx.x < experts ? count[threadIdx.x] : 0, t = (c + tile - 1) / tile, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int before = t;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int a = __shfl_up(before, by);
        if (lane >= by) before += a;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    for (int w = 0; w < wave; w++) before += sums[w];
    if ((int)threadIdx.x < experts) tile_at[threadIdx.x] = before - t;
    if (threadIdx.x == kDealThreads - 1) {  // (experts beyond the last have none, so this thread's sum is all of them)
        tile_at[experts] = before;
        if (blockIdx.x == 0) *tiles_count = before + (count[experts] + tile - 1) / tile;
    }
    if (blockIdx.x == 0) {
        for (int at = 0, i = before - t; (int)threadIdx.x < experts && at < c; at += tile, i++) tiles[i] = {(int)threadIdx.x, c - at < tile ? c - at : tile};
        if (threadIdx.x == kDealThreads - 1)
            for (int at = 0, i = before; at < count[experts]; at += tile, i++) tiles[i] = {-1, count[experts] - at < tile ? count[experts] - at : tile};
    }
    __syncthreads();
    const auto place = [&](int i, int e) { order[tile_at[e] * tile + atomicAdd(&first[e], 1)] = i; };
    each_of(mine, place);
    for (int i = begin + threadIdx.x + kPairsAhead * kDealThreads; i < end; i += kPairsAhead * kDealThreads) each_of(pairs_of(ids, i, end, experts), place);
}

// out[t] = sum over j, ascending, of weights[t][j] products[t][j].  Four columns a lane, the rows of eight choices on their way at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_join_kernel(const float *products, const int *ids, const float *weights, int64_t tokens, int choices, int experts,
                                                               int N, T *out) {
    constexpr int kAhead = 8;
    struct __attribute__((packed, aligned(4))) Four {
        float v[4];
    };
    const int64_t t = blockIdx.y + (int64_t)blockIdx.z * 32768;
    const int n = 4 * (int)(blockIdx.x * kThreads + threadIdx.x), left = N - n;
    if (left <= 0 || t >= tokens) return;
    float y[4] = {};
    for (int j0 = 0; j0 < choices; j0 += kAhead) {
        float w[kAhead];
        bool there[kAhead];
        Four p[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            const int64_t pair = t * choices + (j0 + j < choices ? j0 + j : j0);
            const int e = ids[pair];
            there[j] = j0 + j < choices && e >= 0 && e < experts;
            w[j] = weights[pair];
            const float *from = products + pair * N + n;
            if (left >= 4) p[j] = *reinterpret_cast<const Four *>(from);
            else
#pragma unroll
                for (int c = 0; c < 4; c++) p[j].v[c] = c < left ? from[c] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kAhead; j++)
#pragma unroll
            for (int c = 0; c < 4; c++) y[c] = there[j] ? fmaf(w[j], p[j].v[c], y[c]) : y[c];
    }
    store_any<4, false>(out + t * N + n, left, y);
}

}  // namespace

hipError_t launch_linear_deal(const int *ids, int pairs, int experts, int tile, int *counts, int *tiles_count, Tile *tiles, int *order, hipStream_t s) {
    const int parts = deal_parts(pairs), per_part = (pairs + parts - 1) / parts;
    if (parts > 1) linear_count_kernel<<<parts, kDealThreads, 0, s>>>(ids, pairs, per_part, experts, counts);
    linear_deal_kernel<<<parts, kDealThreads, 0, s>>>(ids, pairs, per_part, experts, tile, parts > 1 ? counts : nullptr, tiles_count, tiles, order);
    return hipGetLastError();
}

hipError_t launch_linear_join(const float *products, const int *ids, const float *weights, int64_t tokens, int choices, int experts, int N, int dtype, void *out,
                              hipStream_t s) {
    const dim3 grid((N + 4 * kThreads - 1) / (4 * kThreads), (unsigned)std::min<int64_t>(tokens, 32768), (unsigned)((tokens + 32767) / 32768));
    if (dtype == BIFEAT_F32) linear_join_kernel<<<grid, kThreads, 0, s>>>(products, ids, weights, tokens, choices, experts, N, (float *)out);
    else if (dtype == BIFEAT_F16) linear_join_kernel<<<grid, kThreads, 0, s>>>(products, ids, weights, tokens, choices, experts, N, (Half16 *)out);
    else linear_join_kernel<<<grid, kThreads, 0, s>>>(products, ids, weights, tokens, choices, experts, N, (Brain16 *)out);
    return hipGetLastError();
}

}  // namespace bf
