// Tokens routed to experts: scores, ranks, the choice and its weights, and the logits' gradient.
#include <math.h>

#include <type_traits>

#include "cache.hpp"

#define BF_HIP(call)                                                   \
    do {                                                               \
        hipError_t e_ = (call);                                        \
        if (e_ != hipSuccess) return bf::record_hip_error(e_, #call);  \
    } while (0)

namespace bf {
namespace {

// A wave takes a token, a lane EPL neighbouring experts.  Where ranks are the logits alone, they are 32-bit numbers, and scores are needed of the chosen only.
// Where scores count (a bias, sums of groups, softmax without shares) they and ranks are 64-bit numbers: which of two experts is before the other may hang
// on the last digits, and ranks in 32 bits would put another one first in 3 of 100 000 choices of 8 among 256.
constexpr int kTokensAtOnce = kThreads / 64;

struct Options {
    int experts, choices, groups, top_groups;
    bool sigmoid, two, renormalise;
    double scale;
    const float *bias;
    int lanes_log2;  // of a group, where it is whole lanes and a power of two of them; else -1
};

// ---- over a wave's lanes, without LDS: by moves within rows of 16, then from row to row; the result in the last lane
template <int CTRL, int ROWS>
__device__ inline uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ inline double moved(double x) {
    const uint2 w = __builtin_bit_cast(uint2, x);
    return __builtin_bit_cast(double, make_uint2(moved<CTRL, ROWS>(w.x), moved<CTRL, ROWS>(w.y)));
}
template <typename X, typename F>
__device__ inline X over_wave(X x, F f) {
    x = f(x, moved<0x111, 0xf>(x));  // the lane below
    x = f(x, moved<0x112, 0xf>(x));  // two below, four, eight
    x = f(x, moved<0x114, 0xf>(x));
    x = f(x, moved<0x118, 0xf>(x));
    x = f(x, moved<0x142, 0xa>(x));  // the last of the row below, in every other row
    x = f(x, moved<0x143, 0xc>(x));  // the last of the lower half
    return x;
}
__device__ inline uint32_t of_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
__device__ inline double of_lane(double x, int lane) {
    const uint2 w = __builtin_bit_cast(uint2, x);
    return __builtin_bit_cast(double, make_uint2(of_lane(w.x, lane), of_lane(w.y, lane)));
}
__device__ inline uint32_t wave_most(uint32_t x) {
    return of_lane(over_wave(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), 63);
}
__device__ inline double wave_sum(double x) {
    return of_lane(over_wave(x, [](double a, double b) { return a + b; }), 63);
}

// ---- ranks as whole numbers in the same order; 0: not to be had
__device__ inline uint32_t key_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return x > -INFINITY ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;  // (a NaN is not)
}
__device__ inline uint64_t key_of(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return x > -INFINITY ? (b >> 63 ? ~b : b | 1ull << 63) : 0ull;
}
__device__ inline float of_key(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// (0 and -0 are equal)
__device__ inline float plain_zero(float x) { return x == 0.f ? 0.f : x; }

// The first lane that holds the largest key, and its upper 32 bits, the same in all lanes; 0 of them: no lane has one.
__device__ inline int first_best(uint32_t key, uint32_t &most) {
    most = wave_most(key);
    return __builtin_ctzll(__ballot(key == most));
}
__device__ inline int first_best(uint64_t key, uint32_t &most) {
    const uint32_t high = (uint32_t)(key >> 32);
    most = wave_most(high);
    uint64_t which = __ballot(high == most);
    if (which & (which - 1)) {
        const uint32_t low = high == most ? (uint32_t)key : 0u;
        const uint32_t rest = wave_most(low);
        which = __ballot(high == most && low == rest);
    }
    return __builtin_ctzll(which);
}

// A lane's logits, -infinity past the last expert; true in `spoilt` where the token's weights are NaN.
template <typename T, int EPL>
__device__ inline void logits_of(const T *row, const Options &o, int lane, float (&x)[EPL], bool &spoilt) {
    const int e0 = lane * EPL;
    if (e0 + EPL <= o.experts) {
        struct __attribute__((packed, aligned(sizeof(T)))) Logits {
            T v[EPL];
        };
        const Logits l = *reinterpret_cast<const Logits *>(row + e0);
#pragma unroll
        for (int i = 0; i < EPL; i++) x[i] = to_float(l.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < EPL; i++) x[i] = e0 + i < o.experts ? to_float(row[e0 + i]) : -INFINITY;
    }
    bool nan = false;
#pragma unroll
    for (int i = 0; i < EPL; i++) {
        x[i] = plain_zero(x[i]);
        nan |= x[i] != x[i] || (!o.sigmoid && x[i] == INFINITY);
    }
    spoilt = __ballot(nan) != 0;
}

__device__ inline double sigmoid(float x) { return 1.0 / (1.0 + exp(-(double)x)); }

// All scores.
template <int EPL>
__device__ inline void scores_of(const float (&x)[EPL], const Options &o, double (&score)[EPL]) {
    if (o.sigmoid) {
#pragma unroll
        for (int i = 0; i < EPL; i++) score[i] = sigmoid(x[i]);
        return;
    }
    uint32_t key = 0;
#pragma unroll
    for (int i = 0; i < EPL; i++) key = key_of(x[i]) > key ? key_of(x[i]) : key;
    key = wave_most(key);
    const double most = key ? (double)of_key(key) : 0.0;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; i++) {
        score[i] = exp((double)x[i] - most);
        sum += score[i];
    }
    sum = wave_sum(sum);
    const double inverse = sum != 0.0 ? 1.0 / sum : 0.0;  // (all masked: no expert has a score)
#pragma unroll
    for (int i = 0; i < EPL; i++) score[i] *= inverse;
}

// The experts that the kept groups do not hold are no longer to be had.  worth: what counts of an expert for its group.
template <int EPL, typename Key>
__device__ inline void keep_groups(const Options &o, int lane, double *room, Key (&key)[EPL], const double (&worth)[EPL]) {
    const int per = o.experts / o.groups;
    // (a group's worth is a key again: of its best expert, or of the sum of two)
    if (o.lanes_log2 >= 0) {
        const int lanes = 1 << o.lanes_log2;
        Key of_group = 0;
        if (!o.two) {
#pragma unroll
            for (int i = 0; i < EPL; i++) of_group = key[i] > of_group ? key[i] : of_group;
            for (int by = 1; by < lanes; by *= 2) {
                const Key other = __shfl_xor(of_group, by);
                of_group = other > of_group ? other : of_group;
            }
        } else if constexpr (sizeof(Key) == 8) {
            double best = -INFINITY, second = -INFINITY;
#pragma unroll
            for (int i = 0; i < EPL; i++) {
                const double w = key[i] ? worth[i] : -INFINITY;
                second = fmax(second, fmin(best, w));
                best = fmax(best, w);
            }
            for (int by = 1; by < lanes; by *= 2) {
                const double b = __shfl_xor(best, by), s = __shfl_xor(second, by);
                second = fmax(fmin(best, b), fmax(second, s));
                best = fmax(best, b);
            }
            of_group = key_of(second > -INFINITY ? best + second : best);
        }
        bool kept = false;
        for (int j = 0; j < o.top_groups; j++) {
            uint32_t most;
            const int first = first_best(of_group, most);
            if (most == 0) break;
            if (lane >> o.lanes_log2 == first >> o.lanes_log2) kept = true, of_group = 0;
        }
#pragma unroll
        for (int i = 0; i < EPL; i++) key[i] = kept ? key[i] : 0;
        return;
    }
    // groups that lie across lanes, by way of LDS: a lane takes a group
    if constexpr (sizeof(Key) == 8) {
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (lane * EPL + i < o.experts) room[lane * EPL + i] = key[i] ? worth[i] : -INFINITY;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        double best = -INFINITY, second = -INFINITY;
        if (lane < o.groups)
            for (int i = 0; i < per; i++) {
                const double w = room[lane * per + i];
                second = fmax(second, fmin(best, w));
                best = fmax(best, w);
            }
        uint64_t of_group = key_of(o.two && second > -INFINITY ? best + second : best), kept = 0;
        for (int j = 0; j < o.top_groups; j++) {
            uint32_t most;
            const int g = first_best(of_group, most);
            if (most == 0) break;
            kept |= 1ull << g;
            if (lane == g) of_group = 0;
        }
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (!(kept >> ((lane * EPL + i) / per & 63) & 1)) key[i] = 0;
    }
}

// WIDE: ranks and scores are 64-bit numbers (see the top).
template <typename T, int EPL, bool WIDE>
__global__ __launch_bounds__(kThreads) void route_kernel(const T *logits, int64_t stride, int64_t tokens, Options o, int *ids, float *weights) {
    typedef std::conditional_t<WIDE, uint64_t, uint32_t> Key;
    extern __shared__ double ranks[];  // [token of the workgroup][expert], where groups lie across lanes
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t t = (int64_t)blockIdx.x * kTokensAtOnce + wave;
    if (t >= tokens) return;
    float x[EPL];
    bool spoilt;
    logits_of<T, EPL>(logits + t * stride, o, lane, x, spoilt);
    Key key[EPL];
    double score[EPL];
    if constexpr (WIDE) {
        double worth[EPL];
        scores_of<EPL>(x, o, score);
#pragma unroll
        for (int i = 0; i < EPL; i++) {
            const int e = lane * EPL + i;
            const bool there = e < o.experts && x[i] > -INFINITY;
            worth[i] = o.bias && there ? score[i] + (double)o.bias[e] : score[i];
            const double rank = o.bias ? worth[i] : (double)x[i];
            key[i] = there ? key_of(rank) : 0ull;
            if (!o.bias && !o.two) worth[i] = rank;
        }
        if (o.groups > 1) keep_groups<EPL>(o, lane, ranks + wave * o.experts, key, worth);
    } else {
#pragma unroll
        for (int i = 0; i < EPL; i++) key[i] = key_of(x[i]);  // (past the last expert: 0)
        if (o.groups > 1) keep_groups<EPL>(o, lane, nullptr, key, score);
    }
    int id = -1;  // the lane's choice, and its score
    double chosen = 0.0;
    for (int j = 0; j < o.choices; j++) {
        Key best = 0;
        int which = 0;
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (key[i] > best) best = key[i], which = i;
        uint32_t most;
        const int first = first_best(best, most);
        if (most == 0) break;
        const int e = (int)of_lane((uint32_t)(lane * EPL + which), first);
        double its = 0.0;
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < EPL; i++) its = which == i ? score[i] : its;
            its = of_lane(its, first);
        } else {
            its = (double)of_key(most);  // (the logit, for now)
        }
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (lane == first && which == i) key[i] = 0;
        if (lane == j) id = e, chosen = its;
    }
    if constexpr (!WIDE) {
        // the first choice has the largest logit of all, so that shares of softmax scores are shares of exp(x - x_first)
        const double most = of_lane(chosen, 0);
        if (o.sigmoid) chosen = id < 0 ? 0.0 : sigmoid((float)chosen);
        else chosen = id < 0 ? 0.0 : exp(chosen - most);
    }
    double w = o.scale * chosen;
    if (o.renormalise) {
        const double total = wave_sum(chosen);
        w = total > 0.0 ? w / total : 0.0;
    }
    if (lane < o.choices) {
        ids[t * o.choices + lane] = id;
        weights[t * o.choices + lane] = spoilt ? NAN : id < 0 ? 0.f : (float)w;
    }
}

// With g the gradient of the weights, c the scale, s the scores, S their sum over the chosen ones and q_j = s_j / S:
//   softmax, renormalised    dx_i = c q_i (g_i - sum_j g_j q_j) for the chosen, else 0
//   softmax                  dx_i = c s_i ([i chosen] g_i - sum_j g_j s_j)
//   sigmoid, renormalised    dx_i = c q_i (1 - s_i) (g_i - sum_j g_j q_j) for the chosen, else 0
//   sigmoid                  dx_i = c s_i (1 - s_i) g_i for the chosen, else 0
// Lane j has choice j; but for the second of these only the chosen scores are needed, and of the first the largest logit.
template <typename T, int EPL>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(const T *logits, int64_t stride, int64_t tokens, Options o, const int *ids, const float *grad,
                                                                  T *out) {
    const int lane = threadIdx.x % 64;
    const int64_t t = (int64_t)blockIdx.x * kTokensAtOnce + threadIdx.x / 64;
    if (t >= tokens) return;
    int id = -1;
    double g = 0.0;
    float its = -INFINITY;
    if (lane < o.choices) {
        id = ids[t * o.choices + lane];
        if (id < 0 || id >= o.experts) id = -1;
        if (id >= 0) {
            g = grad[t * o.choices + lane];
            its = to_float(logits[t * stride + id]);
        }
    }
    float x[EPL];
    bool spoilt;
    logits_of<T, EPL>(logits + t * stride, o, lane, x, spoilt);
    double all[EPL], d = 0.0, sum = 0.0;
    const bool every = !o.sigmoid && !o.renormalise;
    if (every) {
        scores_of<EPL>(x, o, all);
        for (int j = 0; j < o.choices; j++) {
            const int e = (int)of_lane((uint32_t)id, j);
            const double gj = of_lane(g, j);
#pragma unroll
            for (int i = 0; i < EPL; i++)
                if (e == lane * EPL + i) sum += gj * all[i];
        }
        sum = wave_sum(sum);
    } else {
        double s;
        if (o.sigmoid) {
            s = id >= 0 ? sigmoid(its) : 0.0;
        } else {
            // (beside the largest logit of all, not of the chosen: scores that are 0 have weights of 0, and no gradient)
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < EPL; i++) most = key_of(x[i]) > most ? key_of(x[i]) : most;
            most = wave_most(most);
            s = id >= 0 && most ? exp((double)its - (double)of_key(most)) : 0.0;
        }
        double q = s;
        if (o.renormalise) {
            const double total = wave_sum(s);
            q = total > 0.0 ? s / total : 0.0;
            sum = wave_sum(g * q);
        }
        d = o.scale * q * (g - sum) * (o.sigmoid ? 1.0 - s : 1.0);
    }
    float y[EPL];
#pragma unroll
    for (int i = 0; i < EPL; i++) y[i] = every ? (float)(o.scale * all[i] * -sum) : 0.f;
    for (int j = 0; j < o.choices; j++) {
        const int e = (int)of_lane((uint32_t)id, j);
        const double one = of_lane(every ? g : d, j);
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (e == lane * EPL + i) y[i] = every ? (float)(o.scale * all[i] * (one - sum)) : (float)one;
    }
#pragma unroll
    for (int i = 0; i < EPL; i++) y[i] = spoilt ? NAN : y[i];
    const int e0 = lane * EPL;
    T *to = out + t * o.experts + e0;
    if (e0 + EPL <= o.experts) {
        struct __attribute__((packed, aligned(sizeof(T)))) Logits {
            T v[EPL];
        } l;
#pragma unroll
        for (int i = 0; i < EPL; i++) l.v[i] = from_float<T>(y[i]);
        *reinterpret_cast<Logits *>(to) = l;
    } else {
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (e0 + i < o.experts) to[i] = from_float<T>(y[i]);
    }
}

template <typename T, int EPL>
void route(const void *logits, int64_t stride, int64_t tokens, Options o, int *ids, float *weights, hipStream_t s) {
    const unsigned grid = (unsigned)((tokens + kTokensAtOnce - 1) / kTokensAtOnce);
    o.lanes_log2 = -1;
    const int per = o.experts / o.groups;
    if (per % EPL == 0 && (per / EPL & (per / EPL - 1)) == 0) o.lanes_log2 = ilog2(per / EPL);
    const bool across = o.groups > 1 && o.lanes_log2 < 0;
    const size_t room = across ? sizeof(double) * kTokensAtOnce * o.experts : 0;
    const bool wide = o.bias || across || (!o.sigmoid && !o.renormalise) || (o.groups > 1 && o.two);
    if (wide) route_kernel<T, EPL, true><<<grid, kThreads, room, s>>>((const T *)logits, stride, tokens, o, ids, weights);
    else route_kernel<T, EPL, false><<<grid, kThreads, 0, s>>>((const T *)logits, stride, tokens, o, ids, weights);
}
template <typename T, int EPL>
void route_backward(const void *logits, int64_t stride, int64_t tokens, const Options &o, const int *ids, const float *grad, void *out, hipStream_t s) {
    route_backward_kernel<T, EPL><<<(unsigned)((tokens + kTokensAtOnce - 1) / kTokensAtOnce), kThreads, 0, s>>>((const T *)logits, stride, tokens, o, ids, grad, (T *)out);
}

#define BF_BY_EXPERTS(CALL, T, ...)                              \
    if (o.experts <= 64) CALL<T, 1>(__VA_ARGS__);                \
    else if (o.experts <= 128) CALL<T, 2>(__VA_ARGS__);          \
    else if (o.experts <= 256) CALL<T, 4>(__VA_ARGS__);          \
    else if (o.experts <= 512) CALL<T, 8>(__VA_ARGS__);          \
    else CALL<T, 16>(__VA_ARGS__);
#define BF_BY_TYPE(CALL, ...)                                                    \
    if (dtype == BIFEAT_F32) { BF_BY_EXPERTS(CALL, float, __VA_ARGS__) }         \
    else if (dtype == BIFEAT_F16) { BF_BY_EXPERTS(CALL, Half16, __VA_ARGS__) }   \
    else { BF_BY_EXPERTS(CALL, Brain16, __VA_ARGS__) }

bool options_ok(const bifeat_route_options *o, int32_t dtype, int64_t tokens, int64_t stride) {
    if (!o || (dtype != BIFEAT_F32 && dtype != BIFEAT_F16 && dtype != BIFEAT_BF16)) return false;
    if (o->experts < 1 || o->experts > 1024 || o->choices < 1 || o->choices > 64 || o->choices > o->experts) return false;
    if (o->groups < 1 || o->groups > 64 || o->experts % o->groups || o->top_groups < 1 || o->top_groups > o->groups) return false;
    if ((uint32_t)o->sigmoid > 1 || (uint32_t)o->group_two > 1 || (uint32_t)o->renormalise > 1 || !isfinite(o->scale) || (uintptr_t)o->bias % 4) return false;
    return tokens >= 0 && tokens <= INT32_MAX / 64 && stride >= 0;
}
Options options_of(const bifeat_route_options *o) {
    return {o->experts, o->choices, o->groups, o->top_groups, o->sigmoid != 0, o->group_two != 0, o->renormalise != 0, o->scale, o->bias, -1};
}

}  // namespace
}  // namespace bf

extern "C" {

int bifeat_route(const void *logits, int64_t row_stride, int32_t dtype, int64_t tokens, const bifeat_route_options *options, int32_t *ids,
                 float *weights, void *stream) {
    if (!bf::options_ok(options, dtype, tokens, row_stride)) return BIFEAT_EINVAL;
    if (tokens == 0) return BIFEAT_OK;
    const uintptr_t esz = dtype == BIFEAT_F32 ? 4 : 2;
    if (!logits || (uintptr_t)logits % esz || !ids || (uintptr_t)ids % 4 || !weights || (uintptr_t)weights % 4) return BIFEAT_EINVAL;
    const bf::Options o = bf::options_of(options);
    using namespace bf;
    BF_BY_TYPE(route, logits, row_stride, tokens, o, ids, weights, (hipStream_t)stream)
    BF_HIP(hipGetLastError());
    return BIFEAT_OK;
}

int bifeat_route_backward(const void *logits, int64_t row_stride, int32_t dtype, int64_t tokens, const bifeat_route_options *options,
                          const int32_t *ids, const float *grad_weights, void *grad_logits, void *stream) {
    if (!bf::options_ok(options, dtype, tokens, row_stride)) return BIFEAT_EINVAL;
    if (tokens == 0) return BIFEAT_OK;
    const uintptr_t esz = dtype == BIFEAT_F32 ? 4 : 2;
    if (!logits || (uintptr_t)logits % esz || !ids || (uintptr_t)ids % 4 || !grad_weights || (uintptr_t)grad_weights % 4 || !grad_logits ||
        (uintptr_t)grad_logits % esz)
        return BIFEAT_EINVAL;
    const bf::Options o = bf::options_of(options);
    using namespace bf;
    BF_BY_TYPE(route_backward, logits, row_stride, tokens, o, ids, grad_weights, grad_logits, (hipStream_t)stream)
    BF_HIP(hipGetLastError());
    return BIFEAT_OK;
}

}  // extern "C"
