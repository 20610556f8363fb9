// The paged cache: what its translation units share.
#pragma once

#include <mutex>
#include <type_traits>

#include "common.hpp"

struct bifeat_cache {
    bifeat_cache_spec spec{};
    int rb = 0;              // bytes of a row of codes
    int64_t head_bytes = 0;  // bytes of a page's block of one head
    int64_t page_bytes = 0;
    int opt_validate = 0;
    // what bifeat_cache_attend leaves of contexts that several workgroups share (see cache_attend.hpp): each stream has its own, so that calls on
    // different streams do not meet, and captured calls have one, whichever stream they are replayed on.  Streams of one capture may be branches
    // that are replayed side by side: the first that asks has it
    struct Workspace {
        int device;
        hipStream_t stream;
        bool captured;
        unsigned long long capture;  // the last that asked for it
        float *partial;
        Workspace *next;
    };
    Workspace *workspaces = nullptr;
    std::mutex mutex;  // of the list, and of a call's kernel and join: threads that share a stream enqueue them in turn
};

namespace bf {

int record_hip_error(hipError_t e, const char *what);
int take_block(void **out);  // a device block of 1 KB from a pool, its bytes as the last use left them, and back
void give_block(void *blk);

// The pages as the kernels see them.
struct CachePages {
    uint8_t *pages;
    int64_t head_bytes, page_bytes;
    int heads, d, rb, ps_log2;
    // offsets in a head's block
    __host__ __device__ int ps() const { return 1 << ps_log2; }
    __host__ __device__ int64_t codes(int which) const { return (int64_t)which * rb << ps_log2; }
    __host__ __device__ int64_t floats(int which) const { return ((int64_t)2 * rb << ps_log2) + ((int64_t)8 * which << ps_log2); }
    __device__ uint8_t *block(int page, int head) const { return pages + (int64_t)page * page_bytes + (int64_t)head * head_bytes; }
};

struct CacheBatch {
    const int32_t *tables;
    const int64_t *lengths, *indptr;
    int64_t width, tokens;
    int B;
    int n;  // new tokens of every sequence where indptr is null

    __device__ int64_t first(int b) const { return indptr ? indptr[b] : (int64_t)b * n; }
    __device__ int64_t count(int b) const { return indptr ? indptr[b + 1] - indptr[b] : n; }
    // (a length past the table's room would lead past the table)
    __device__ int64_t length(int b, int ps_log2) const {
        const int64_t l = lengths[b], room = width << ps_log2;
        return l < 0 ? 0 : l > room ? room : l;
    }
};

// The sequence that token t belongs to; the same t in all lanes.  64 offsets a step.
__device__ inline int sequence_of(const CacheBatch &c, int64_t t) {
    if (!c.indptr) return (int)(t / c.n);
    int lo = 0, hi = c.B;  // indptr[lo] <= t < indptr[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, i = lo + (int)(threadIdx.x & 63) * step;
        const int at = __popcll(__ballot(i < hi && c.indptr[i < hi ? i : lo] <= t)) - 1;
        lo += (at > 0 ? at : 0) * step;  // (never below it, whatever the offsets hold)
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

// ---- elements of the three types
struct Half16 { uint16_t bits; };
struct Brain16 { uint16_t bits; };
__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(Half16 x) { return (float)__builtin_bit_cast(_Float16, x.bits); }
__device__ inline float to_float(Brain16 x) { return __builtin_bit_cast(float, (uint32_t)x.bits << 16); }
template <typename T> __device__ inline T from_float(float x);
template <> __device__ inline float from_float<float>(float x) { return x; }
template <> __device__ inline Half16 from_float<Half16>(float x) { return {__builtin_bit_cast(uint16_t, (_Float16)x)}; }
template <> __device__ inline Brain16 from_float<Brain16>(float x) { return {__builtin_bit_cast(uint16_t, (__bf16)x)}; }

// 8 columns of a row at any address, those from `left` on as zeros
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight { T v[8]; };
template <typename T>
__device__ inline void load8_any(const T *p, int left, float (&x)[8]) {
    if (left >= 8) {
        const Eight<T> e = *reinterpret_cast<const Eight<T> *>(p);
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = to_float(e.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i < left ? to_float(p[i]) : 0.f;
    }
}
// Eight columns of a row as they lie in memory.
template <typename T>
struct Columns {
    uint32_t w[2 * sizeof(T)];
};
template <typename T>
__device__ inline Columns<T> load_columns(const T *p) {
    Columns<T> c;
    const Eight<T> e = *reinterpret_cast<const Eight<T> *>(p);
    __builtin_memcpy(c.w, &e, sizeof(c));
    return c;
}
// ... of a row of K < 8 columns, the others as zeros.
template <typename T>
__device__ inline Columns<T> load_short_columns(const T *row, int K) {
    Columns<T> c;
    T v[8] = {};
#pragma unroll
    for (int i = 0; i < 7; i++)
        if (i < K) v[i] = row[i];
    __builtin_memcpy(c.w, v, sizeof(c));
    return c;
}
template <typename T>
__device__ inline Columns<T> no_columns() {
    Columns<T> c;
#pragma unroll
    for (uint32_t &w : c.w) w = 0;
    return c;
}
// N columns next to each other, of which the row has `left`.  STREAMED: not kept in the caches
template <int N, bool STREAMED, typename T>
__device__ inline void store_any(T *p, int left, const float *x) {
    if (left >= N) {
        struct Columns {
            T v[N];
        } e;
#pragma unroll
        for (int i = 0; i < N; i++) e.v[i] = from_float<T>(x[i]);
        typedef uint32_t Words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
        const Words w = __builtin_bit_cast(Words, e);
        if constexpr (STREAMED) __builtin_nontemporal_store(w, reinterpret_cast<Words *>(p));
        else *reinterpret_cast<Words *>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
            if (i < left) p[i] = from_float<T>(x[i]);
    }
}

constexpr int kMostPositions = 1 << 30;  // of a sequence: positions, and their differences, are 32-bit numbers in the kernels

struct HeadRows {
    const void *data;
    int64_t token_stride, head_stride;
};

struct AttendCall {
    CachePages c;
    CacheBatch b;
    HeadRows q;
    int group;  // query heads a cached head
    int dtype;
    float scale, softcap;
    int window;  // 0: none; at most kMostPositions
    const int64_t *prefix;
    const float *slopes;
    void *out;
    hipStream_t s;
};

struct AppendCall {
    HeadRows q;
    int query_heads;  // 0: no queries
    HeadRows k, v;
    int bits, dtype;
    const float *frequencies;
    int pairs;
    bool interleaved;
    double scale;
    void *out;
    hipStream_t s;
};

hipError_t launch_cache_append(const CachePages &c, const CacheBatch &b, const AppendCall &a);
hipError_t launch_cache_write(const CachePages &c, const CacheBatch &b, const HeadRows &k, const HeadRows &v, int bits, int dtype,
                              hipStream_t s);
hipError_t launch_cache_read(const CachePages &c, const CacheBatch &b, void *k, void *v, int bits, int dtype, hipStream_t s);
hipError_t launch_cache_attend(bifeat_cache *h, const AttendCall &a);
void launch_cache_check(const CacheBatch &b, int ps_log2, int64_t num_pages, int32_t *d_bad, hipStream_t s);
// The workspace of calls on `s`, or of captured calls; both are allocated unless `s` is being captured.  Null: there is none.  The handle's mutex is held.
float *workspace_of(bifeat_cache *h, hipStream_t s);

}  // namespace bf
