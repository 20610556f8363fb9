// Attention over the paged cache: which kernel, how many workgroups, and the join of what several of them did of one item.
#include <algorithm>

#include "cache_attend.hpp"

namespace bf {
namespace {

constexpr int kCUs = 256;
constexpr int kRowsWorkgroups = 3 * kCUs, kChunkWorkgroups = 2 * kCUs;  // as many as run at a time

// One workgroup a query row of an item that was shared: its parts are those of the workgroups [w0, w1], each with sums about a
// maximum of its own.
template <int R, int TOK>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendCall a, AttendPlan plan, int dp) {
    __shared__ float weight[1024], red[8];
    __shared__ float part[4][256];
    __shared__ int sh[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = blockIdx.x % R, item = (int)(blockIdx.x / R % plan.items), head = (int)(blockIdx.x / R / plan.items);
    // the item's sequence, and the units of the head's items before it
    const int seq = sequence_of_item<R>(a, item);
    const int rt = item - first_item<R>(a, seq);
    const View v = view_of<R, TOK>(a, seq, rt);
    const int rows = v.n * a.group;
    if (v.units == 0 || rt * R + r >= rows) return;
    const int per = (plan.items + 255) / 256, i0 = tid * per, i1 = i0 + per < plan.items ? i0 + per : plan.items;
    int sum = 0, before = 0;
    if (i0 < i1) {
        int s = sequence_of_item<R>(a, i0);
        int next = first_item<R>(a, s + 1);
        for (int i = i0; i < i1; i++) {
            while (i >= next && s + 1 < a.b.B) next = first_item<R>(a, ++s + 1);
            const int u = view_of<R, TOK>(a, s, i - first_item<R>(a, s)).units;
            sum += u;
            if (i < item) before += u;
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m), before += __shfl_xor(before, m);
    if (lane == 0) sh[wave] = sum, sh[4 + wave] = before;
    __syncthreads();
    const int64_t total = (int64_t)sh[0] + sh[1] + sh[2] + sh[3];
    const int64_t u0 = total * head + sh[4] + sh[5] + sh[6] + sh[7], u1 = u0 + v.units - 1, all = total * a.c.heads;
    const int64_t nw = all < plan.nw ? all : plan.nw;
    const int w0 = (int)(((u0 + 1) * nw - 1) / all), w1 = (int)(((u1 + 1) * nw - 1) / all);
    if (w0 == w1) return;  // one workgroup had it all
    const int64_t stride = R * (dp + 2);
    auto at = [&](int w) { return plan.partial + ((int64_t)w * 2 + (w == w0)) * stride + (int64_t)r * (dp + 2); };
    float top = kNothing;
    for (int w = w0 + tid; w <= w1; w += 256) top = fmaxf(top, at(w)[dp]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) red[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    // weights of 1024 parts at a time; each wave every fourth part, a lane 4 columns (d <= 256)
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, den = 0.f;
    for (int from = w0; from <= w1; from += 1024) {
        const int to = from + 1024 <= w1 ? from + 1024 : w1 + 1;
        __syncthreads();
        for (int w = from + tid; w < to; w += 256) {
            const float e = __builtin_amdgcn_exp2f(at(w)[dp] - top);
            weight[w - from] = e;
            den += e * at(w)[dp + 1];
        }
        __syncthreads();
        for (int w = from + wave; w < to; w += 4) {
            const float e = weight[w - from];
            const float *x = at(w);
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (lane + 64 * k < a.c.d) acc[k] += e * x[lane + 64 * k];
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) den += __shfl_xor(den, m);
    if (lane == 0) red[4 + wave] = den;
#pragma unroll
    for (int k = 0; k < 4; k++) part[wave][lane + 64 * k] = acc[k];
    __syncthreads();
    den = red[4] + red[5] + red[6] + red[7];
    const int row = rt * R + r;
    const int64_t dst = ((a.b.first(seq) + row / a.group) * ((int64_t)a.c.heads * a.group) + head * a.group + row % a.group) * a.c.d;
    if (tid < a.c.d) store_result(a, dst + tid, den != 0.f ? (part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid]) / den : 0.f);
}

template <int R, int TOK>
void launch_join(const AttendCall &a, const AttendPlan &p, int dp) {
    attend_join_kernel<R, TOK><<<(unsigned)((int64_t)p.items * a.c.heads * R), 256, 0, a.s>>>(a, p, dp);
}

// numbers of a head's items, an upper bound where the batch is ragged
int items_of(const AttendCall &a, int R) {
    if (a.b.indptr) return (int)(a.b.tokens * a.group / R) + a.b.B;
    return a.b.B * ((a.b.n * a.group + R - 1) / R);
}

constexpr size_t kPartialFloats =
    2 * 258 * std::max((size_t)kRowsWorkgroups * kRowsR, (size_t)kChunkWorkgroups * 64 * kChunkNT);

}  // namespace

template <int BITS>
hipError_t attend_chunk_bits(const AttendCall &a, const AttendPlan &p, int dp);
static hipError_t launch_attend_chunk(const AttendCall &a, const AttendPlan &p, int bits, int dp) {
    return bits == 8 ? attend_chunk_bits<8>(a, p, dp) : attend_chunk_bits<4>(a, p, dp);
}

bool ensure_partial(bifeat_cache *h, hipStream_t s) {
    if (h->d_partial) return true;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &status) != hipSuccess || status != hipStreamCaptureStatusNone) return false;
    void *p = nullptr;
    if (hipMalloc(&p, sizeof(float) * kPartialFloats) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    h->d_partial = (float *)p;
    return true;
}

hipError_t launch_cache_attend(bifeat_cache *h, const AttendCall &a) {
    const int dp = a.c.d <= 64 ? 64 : a.c.d <= 128 ? 128 : 256, bits = h->spec.bits;
    const bool chunk = a.b.tokens * a.group > (int64_t)32 * a.b.B;
    const int R = chunk ? 64 * kChunkNT : kRowsR, tok = !chunk ? kRowsTok : dp == 256 ? 32 : 64;
    AttendPlan p;
    p.items = items_of(a, R);
    const int64_t most = ((a.b.width << a.c.ps_log2) + tok - 1) / tok, all = (int64_t)p.items * a.c.heads;
    // contexts of a few units, and calls that find no workspace: an item a workgroup, nothing to join
    const bool split = most > 4 && ensure_partial(h, a.s);
    p.partial = split ? h->d_partial : nullptr;
    p.nw = (int)(split ? std::min<int64_t>(all * most, chunk ? kChunkWorkgroups : kRowsWorkgroups) : all);
    if (chunk) {
        if (hipError_t e = launch_attend_chunk(a, p, bits, dp)) return e;
        if (split) {
            if (dp == 256) launch_join<64 * kChunkNT, 32>(a, p, dp);
            else launch_join<64 * kChunkNT, 64>(a, p, dp);
        }
    } else {
        launch_attend_rows(a, p, bits, dp);
        if (split) launch_join<kRowsR, kRowsTok>(a, p, dp);
    }
    return hipGetLastError();
}

}  // namespace bf
