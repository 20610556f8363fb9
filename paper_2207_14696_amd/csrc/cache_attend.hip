// Attention over the paged cache: which kernel, how many workgroups, and the join of what several of them did of one item.
#include <algorithm>
#include <new>

#include "cache_attend.hpp"

namespace bf {
namespace {

constexpr int kCUs = 256;
// workgroups: as many as run at a time
constexpr int rows_workgroups(int dp) { return kCUs * (dp == 64 ? 3 : dp == 128 ? 2 : 1); }
constexpr int chunk_workgroups(int dp, int np) { return kCUs * (dp == 256 && np == 2 ? 1 : 2); }

// Joins the parts of the items that several workgroups have.  Blocks (w, y): the item that workgroup w goes on with, if it is the
// first to go on with it; WAVES waves a query row, 16 lanes a part.  The order of the sums is fixed by the parts' numbers.  A chain
// of two fetches: where the parts are, then all of a part at once.  It waits for them: what 512 workgroups leave of 128 rows of 128 columns
// (68 MB) takes 21 us, of 16 rows 3 to 8.
template <int R, int DP, int WAVES>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendCall a, AttendPlan plan) {
    const int w = blockIdx.x;
    const PartOf b = plan.begins[w];
    if (w >= b.nw || b.unit == 0) return;
    const int first = b.start - b.unit;  // the item's first unit
    if (start_of(w - 1, b.all, b.nw) > first) return;
    // parts: of w - 1, which has its beginning, and of [w, w1]
    const int w1 = workgroup_of(first + b.units - 1, b.all, b.nw);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane & 15;
    constexpr int kGroups = 4 * WAVES, kRows = 4 / WAVES, kC = DP / 64;  // part groups a row, rows at a time, float4s a lane
    const int group = (wave % WAVES) * 4 + lane / 16;
    __shared__ float tops[4], dens[4], part[WAVES > 1 ? 4 : 1][DP];
    const int64_t stride = R * (DP + 2);
    for (int r0 = blockIdx.y * kRows; r0 < b.rows; r0 += gridDim.y * kRows) {
        const bool real = r0 + wave / WAVES < b.rows;
        const int r = real ? r0 + wave / WAVES : b.rows - 1;
        float4 acc[kC];  // columns 64 c + 4 sub
        float den = 0.f, top = kNothing;
#pragma unroll
        for (int c = 0; c < kC; c++) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        auto scale = [&](float by) {
            den *= by;
#pragma unroll
            for (int c = 0; c < kC; c++) acc[c].x *= by, acc[c].y *= by, acc[c].z *= by, acc[c].w *= by;
        };
#pragma unroll 2
        for (int k = w - 1 + group; k <= w1; k += kGroups) {
            const float *x = plan.partial + ((int64_t)k * 2 + (k == w - 1)) * stride;
            const float its = x[R * DP + r], sum = x[R * DP + R + r];
            float4 y[kC];
#pragma unroll
            for (int c = 0; c < kC; c++) y[c] = *reinterpret_cast<const float4 *>(x + r * DP + 64 * c + 4 * sub);
            const float now = fmaxf(top, its), e = __builtin_amdgcn_exp2f(its - now);
            scale(__builtin_amdgcn_exp2f(top - now));
            top = now;
            den = fmaf(e, sum, den);
#pragma unroll
            for (int c = 0; c < kC; c++) {
                acc[c].x = fmaf(e, y[c].x, acc[c].x);
                acc[c].y = fmaf(e, y[c].y, acc[c].y);
                acc[c].z = fmaf(e, y[c].z, acc[c].z);
                acc[c].w = fmaf(e, y[c].w, acc[c].w);
            }
        }
        float all = fmaxf(top, __shfl_xor(top, 16));
        all = fmaxf(all, __shfl_xor(all, 32));
        if constexpr (WAVES > 1) {
            if (lane == 0) tops[wave] = all;
            __syncthreads();
            all = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        }
        scale(__builtin_amdgcn_exp2f(top - all));
#pragma unroll
        for (int m = 16; m < 64; m *= 2) {
            den += __shfl_xor(den, m);
#pragma unroll
            for (int c = 0; c < kC; c++) {
                acc[c].x += __shfl_xor(acc[c].x, m);
                acc[c].y += __shfl_xor(acc[c].y, m);
                acc[c].z += __shfl_xor(acc[c].z, m);
                acc[c].w += __shfl_xor(acc[c].w, m);
            }
        }
        if constexpr (WAVES > 1) {
            if (lane == 0) dens[wave] = den;
            if (lane < 16)
#pragma unroll
                for (int c = 0; c < kC; c++) *reinterpret_cast<float4 *>(&part[wave][64 * c + 4 * sub]) = acc[c];
            __syncthreads();
            den = dens[0] + dens[1] + dens[2] + dens[3];
        }
        const int row = b.rt * R + r;
        const int64_t dst = ((b.token + row / a.group) * ((int64_t)a.c.heads * a.group) + b.head * a.group + row % a.group) * a.c.d;
        const float inv = den != 0.f ? 1.f / den : 0.f;
        if constexpr (WAVES > 1) {
            if (tid < a.c.d) store_result(a, dst + tid, (part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid]) * inv);
            __syncthreads();
        } else if (real && lane < 16) {
#pragma unroll
            for (int c = 0; c < kC; c++) {
                const int col = 64 * c + 4 * sub;
                store_four(a, dst + col, a.c.d - col, make_float4(acc[c].x * inv, acc[c].y * inv, acc[c].z * inv, acc[c].w * inv));
            }
        }
    }
}

// rows: the most that an item has.  Four waves a row where an item of 16 rows may have 48 parts or more (one sequence of 12 288, 4 rows
// on each of 8 heads of 128, 48 parts: the call 18.7 us, with one wave 20.0; of 65 536 on one head, 256 parts: 21.1 and 28.7), one where it has
// fewer (8 sequences of 2048 on 8 heads, 8 parts: 19.1, with four 20.3; two of 8192, 32 parts: 20.1 and 20.7).
template <int R, int WAVES>
void launch_join(const AttendCall &a, const AttendPlan &p, int dp, int rows) {
    const dim3 grid(p.nw, std::min(16, (rows * WAVES + 3) / 4));
    if (dp == 64) attend_join_kernel<R, 64, WAVES><<<grid, 256, 0, a.s>>>(a, p);
    else if (dp == 128) attend_join_kernel<R, 128, WAVES><<<grid, 256, 0, a.s>>>(a, p);
    else attend_join_kernel<R, 256, WAVES><<<grid, 256, 0, a.s>>>(a, p);
}

// numbers of a head's items, an upper bound where the batch is ragged (times heads within an int: see bifeat_cache_attend)
int items_of(const AttendCall &a, int R) {
    if (a.b.indptr) return (int)(a.b.tokens * a.group / R) + a.b.B;
    return a.b.B * ((a.b.n * a.group + R - 1) / R);
}

constexpr size_t kPartialFloats =
    2 * (size_t)chunk_workgroups(128, 1) * 128 * (128 + 2);  // (the most that any kernel's leave: 128 rows of 128 columns)

}  // namespace

template <int BITS>
hipError_t attend_chunk_bits(const AttendCall &a, const AttendPlan &p, int dp);
static hipError_t launch_attend_chunk(const AttendCall &a, const AttendPlan &p, int bits, int dp) {
    return bits == 8 ? attend_chunk_bits<8>(a, p, dp) : attend_chunk_bits<4>(a, p, dp);
}

float *workspace_of(bifeat_cache *h, hipStream_t s) {
    int device = 0;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    unsigned long long capture = 0;
    if (hipGetDevice(&device) != hipSuccess || hipStreamGetCaptureInfo(s, &status, &capture) != hipSuccess) {
        (void)hipGetLastError();
        return nullptr;
    }
    const bool capturing = status != hipStreamCaptureStatusNone;
    auto find = [&](bool captured) {
        bifeat_cache::Workspace *w = h->workspaces;
        while (w && !(w->device == device && w->captured == captured && (captured || w->stream == s))) w = w->next;
        return w;
    };
    if (capturing) {
        bifeat_cache::Workspace *w = find(true);
        if (w && w->capture != capture) w->capture = capture, w->stream = s;
        return w && w->stream == s ? w->partial : nullptr;
    }
    if (const bifeat_cache::Workspace *w = find(false)) return w->partial;
    for (const bool captured : {true, false}) {
        if (find(captured)) continue;
        auto *w = new (std::nothrow) bifeat_cache::Workspace{device, s, captured, 0, nullptr, h->workspaces};
        if (!w) return nullptr;
        if (hipMalloc((void **)&w->partial, sizeof(float) * kPartialFloats + sizeof(PartOf) * rows_workgroups(64)) != hipSuccess) {
            (void)hipGetLastError();
            delete w;
            return nullptr;
        }
        h->workspaces = w;
    }
    return find(false)->partial;
}

hipError_t launch_cache_attend(bifeat_cache *h, const AttendCall &a) {
    const int dp = a.c.d <= 64 ? 64 : a.c.d <= 128 ? 128 : 256, bits = h->spec.bits;
    const int np = a.dtype == BIFEAT_F32 ? 2 : 1;
    const int64_t width = a.b.width << a.c.ps_log2;
    // (an item has one unit at least, also over tables that have no room: its zeros)
    auto units_of = [&](int R, int tok) { return (int64_t)items_of(a, R) * a.c.heads * std::max<int64_t>(1, (width + tok - 1) / tok); };
    // The kernel for many rows makes operands once for 64 or 128 rows; that for few, for 16, starts and joins sooner.  Few: up to 64
    // rows of 64 columns a sequence and head on average (64 sequences of 4096, 12 heads: 294 us, the other kernel 300; 128
    // rows 577 and 310), 32 of 128 (8 heads: 193 and 207; 48 rows 286 and 235), 16 of 256 (4 heads: 20 rows 195 and 161; 32 where a
    // window leaves an unknown part of the context: 20 rows, 1024 positions seen 47 and 64).  And any number where the units
    // come to 10 a workgroup or fewer: 64 rows of 8 sequences of 2048 on 8 heads of 128 (10) 40 and 53, 256 rows of one of 512 (1)
    // 15 and 30, 256 rows of 8 of 1024 (17) 67 and 58.  Not for 32-bit queries, whose operands cost twice (385 rows of three of
    // 1001, 2 units: 32 and 29.5).  Lengths are not known here: a context counts as long as its page table is wide (a token over 300 9.0 us, 16.3 by a table 4 times as wide), and
    // rows are a mean over the batch (2048 rows over 16 384 beside 255 single tokens of 2048, 8 heads of 128: 873 us, in calls of their
    // own 252 and 201).
    const int few = dp == 64 ? 64 : dp == 256 && !a.window ? 16 : 32;
    const bool chunk = a.b.tokens * a.group > (int64_t)few * a.b.B &&
                       (np == 2 || units_of(kRowsR, kRowsTok) > 10 * rows_workgroups(dp));
    const int R = chunk ? 64 * chunk_tiles(dp, np) : kRowsR, tok = !chunk ? kRowsTok : dp == 256 ? 32 : 64;
    const int most = chunk ? chunk_workgroups(dp, np) : rows_workgroups(dp);
    AttendPlan p;
    p.items = items_of(a, R);
    const int64_t all = (int64_t)p.items * a.c.heads, units = units_of(R, tok);
    // An item a workgroup and nothing to join: where the workgroups all run at once and have 6 units or fewer (2 of the kernel for
    // many rows); 4 rows of 8 sequences on 8 heads of 128: at 512 positions 13.6 us, dealt evenly and joined 16.0; at
    // 1024 19.3 and 16.3.  And calls that find no workspace, or have 2^31 units or more.
    const bool small = width <= (chunk ? 128 : 6 * kRowsTok) && all <= most;
    std::unique_lock<std::mutex> lock(h->mutex, std::defer_lock);
    p.partial = nullptr;
    if (!small && units <= INT32_MAX) {
        lock.lock();
        p.partial = workspace_of(h, a.s);
    }
    const bool split = p.partial;
    p.begins = split ? reinterpret_cast<PartOf *>(p.partial + kPartialFloats) : nullptr;
    p.least = !chunk ? 2 : np == 2 ? 1 : 4;
    p.nw = split ? workgroups_of(units, p.least, most) : (int)all;  // (bifeat_cache_attend has seen to it that they fit an int)
    const int rows = a.b.indptr ? R : std::min(R, a.b.n * a.group);
    if (chunk) {
        if (hipError_t e = launch_attend_chunk(a, p, bits, dp)) return e;
        if (split) R == 128 ? launch_join<128, 1>(a, p, dp, rows) : launch_join<64, 1>(a, p, dp, rows);
    } else {
        launch_attend_rows(a, p, bits, dp);
        if (split) p.nw < (int64_t)48 * a.b.B * a.c.heads ? launch_join<kRowsR, 1>(a, p, dp, rows) : launch_join<kRowsR, 4>(a, p, dp, rows);
    }
    return hipGetLastError();
}

}  // namespace bf
