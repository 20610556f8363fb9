// Tokens' choices dealt to the experts that they name, and the experts' products joined.
#include "linear.hpp"

namespace bf {
namespace {

constexpr int kDealThreads = 1024, kMostExperts = 1024;

// Pairs of a token and a choice, expert by expert, and tiles of up to `tile` of one expert's.  The order of an expert's pairs is not fixed; their products do
// not depend on it.  Those that name no expert come last, as an expert of their own.
__global__ __launch_bounds__(kDealThreads) void linear_deal_kernel(const int *ids, int pairs, int experts, int tile, int *tiles_count, Tile *tiles,
                                                                   int *order) {
    __shared__ int count[kMostExperts + 1], first[kMostExperts + 1], tile_at[kMostExperts + 1];
    __shared__ int sums[2][kDealThreads / 64];
    for (int e = threadIdx.x; e <= experts; e += kDealThreads) count[e] = 0;
    __syncthreads();
    const auto expert_of = [&](int i) {
        const int e = ids[i];
        return e >= 0 && e < experts ? e : experts;
    };
    for (int i = threadIdx.x; i < pairs; i += kDealThreads) atomicAdd(&count[expert_of(i)], 1);
    __syncthreads();
    // sums of the pairs and tiles before each expert: a thread an expert, the last with those of none besides
    int c = (int)threadIdx.x < experts ? count[threadIdx.x] : 0, before = c, t = (c + tile - 1) / tile, tiles_before = t;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const int a = __shfl_up(before, by), b = __shfl_up(tiles_before, by);
        if (lane >= by) before += a, tiles_before += b;
    }
    if (lane == 63) sums[0][wave] = before, sums[1][wave] = tiles_before;
    __syncthreads();
    for (int w = 0; w < wave; w++) before += sums[0][w], tiles_before += sums[1][w];
    if ((int)threadIdx.x < experts) first[threadIdx.x] = before - c, tile_at[threadIdx.x] = tiles_before - t;
    if (threadIdx.x == kDealThreads - 1) {  // (experts beyond the last have none, so this thread's sums are all of them)
        first[experts] = before;
        tile_at[experts] = tiles_before;
        *tiles_count = tiles_before + (count[experts] + tile - 1) / tile;
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= experts; e += kDealThreads)
        for (int at = 0, i = tile_at[e]; at < count[e]; at += tile, i++)
            tiles[i] = {e < experts ? e : -1, first[e] + at, count[e] - at < tile ? count[e] - at : tile, 0};
    __syncthreads();
    for (int i = threadIdx.x; i < pairs; i += kDealThreads) order[atomicAdd(&first[expert_of(i)], 1)] = i;
}

// out[t] = sum over j, ascending, of weights[t][j] products[t][j].  Four columns a lane.
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_join_kernel(const float *products, const int *ids, const float *weights, int64_t tokens, int choices, int experts,
                                                               int N, T *out) {
    const int pieces = (N + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < tokens * pieces; i += (int64_t)gridDim.x * kThreads) {
        const int64_t t = i / pieces;
        const int n = 4 * (int)(i - t * pieces), left = N - n;
        float y[4] = {};
        for (int j = 0; j < choices; j++) {
            const int64_t pair = t * choices + j;
            const int e = ids[pair];
            if (e < 0 || e >= experts) continue;
            const float w = weights[pair];
            const float *p = products + pair * N + n;
#pragma unroll
            for (int c = 0; c < 4; c++)
                if (c < left) y[c] = fmaf(w, p[c], y[c]);
        }
        store_any<4, false>(out + t * N + n, left, y);
    }
}

}  // namespace

hipError_t launch_linear_deal(const int *ids, int pairs, int experts, int tile, int *tiles_count, Tile *tiles, int *order, hipStream_t s) {
    linear_deal_kernel<<<1, kDealThreads, 0, s>>>(ids, pairs, experts, tile, tiles_count, tiles, order);
    return hipGetLastError();
}

hipError_t launch_linear_join(const float *products, const int *ids, const float *weights, int64_t tokens, int choices, int experts, int N, int dtype, void *out,
                              hipStream_t s) {
    const int64_t threads = tokens * ((N + 3) / 4);
    const unsigned grid = (unsigned)(threads / kThreads >= (1 << 20) ? 1 << 20 : threads / kThreads + 1);
    if (dtype == BIFEAT_F32) linear_join_kernel<<<grid, kThreads, 0, s>>>(products, ids, weights, tokens, choices, experts, N, (float *)out);
    else if (dtype == BIFEAT_F16) linear_join_kernel<<<grid, kThreads, 0, s>>>(products, ids, weights, tokens, choices, experts, N, (Half16 *)out);
    else linear_join_kernel<<<grid, kThreads, 0, s>>>(products, ids, weights, tokens, choices, experts, N, (Brain16 *)out);
    return hipGetLastError();
}

}  // namespace bf
