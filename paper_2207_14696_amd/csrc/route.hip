// Tokens routed to experts: scores, ranks, the choice and its weights, and the logits' gradient.
#include <math.h>

#include "cache.hpp"

#define BF_HIP(call)                                                   \
    do {                                                               \
        hipError_t e_ = (call);                                        \
        if (e_ != hipSuccess) return bf::record_hip_error(e_, #call);  \
    } while (0)

namespace bf {
namespace {

// A wave takes a token; lane l has experts l, l + 64, ...  Scores, ranks and sums are 64-bit numbers: which of two experts is before the other may hang on the
// last digits, and ranks in 32 bits would put another one first in 3 of 100 000 choices of 8 among 256.
constexpr int kTokensAtOnce = kThreads / 64;

struct Options {
    int experts, choices, groups, top_groups;
    bool sigmoid, two, renormalise;
    double scale;
    const float *bias;
};

__device__ inline double shuffled(double x, int by) { return __shfl_xor(x, by); }
__device__ inline double wave_sum(double x) {
#pragma unroll
    for (int by = 32; by; by /= 2) x += shuffled(x, by);
    return x;
}
// the best of all lanes' ranks, of equal ones the lowest number, in all of them
__device__ inline void wave_best(double &rank, int &number) {
#pragma unroll
    for (int by = 32; by; by /= 2) {
        const double r = shuffled(rank, by);
        const int n = __shfl_xor(number, by);
        if (r > rank || (r == rank && n < number)) rank = r, number = n;
    }
}

// A token's scores; true in `spoilt` where its weights are NaN.
template <typename T, int EPL>
__device__ inline void scores_of(const T *row, const Options &o, int lane, double (&x)[EPL], double (&score)[EPL], bool &spoilt) {
    double most = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < EPL; i++) {
        const int e = lane + 64 * i;
        x[i] = e < o.experts ? (double)to_float(row[e]) : -INFINITY;
        nan |= x[i] != x[i] || (!o.sigmoid && x[i] == INFINITY);
        most = fmax(most, x[i]);
    }
    spoilt = __ballot(nan) != 0;
    if (o.sigmoid) {
#pragma unroll
        for (int i = 0; i < EPL; i++) score[i] = 1.0 / (1.0 + exp(-x[i]));
        return;
    }
#pragma unroll
    for (int by = 32; by; by /= 2) most = fmax(most, shuffled(most, by));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; i++) {
        score[i] = most == -INFINITY ? 0.0 : exp(x[i] - most);  // (all masked: no expert has a score)
        sum += score[i];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < EPL; i++) score[i] = sum != 0.0 ? score[i] / sum : 0.0;
}

template <typename T, int EPL>
__global__ __launch_bounds__(kThreads) void route_kernel(const T *logits, int64_t stride, int64_t tokens, Options o, int *ids, float *weights) {
    extern __shared__ double ranks[];  // [token of the workgroup][expert], with groups
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t t = (int64_t)blockIdx.x * kTokensAtOnce + wave;
    if (t >= tokens) return;
    double x[EPL], score[EPL], rank[EPL];
    bool spoilt;
    scores_of<T, EPL>(logits + t * stride, o, lane, x, score, spoilt);
#pragma unroll
    for (int i = 0; i < EPL; i++) {
        const int e = lane + 64 * i;
        rank[i] = -INFINITY;
        if (e < o.experts && x[i] > -INFINITY) {
            const double r = o.bias ? score[i] + (double)o.bias[e] : x[i];
            rank[i] = r == r ? r : -INFINITY;
        }
    }
    if (o.groups > 1) {
        double *mine = ranks + wave * o.experts;
        const int per = o.experts / o.groups;
#pragma unroll
        for (int i = 0; i < EPL; i++) {
            const int e = lane + 64 * i;
            if (e < o.experts) mine[e] = !o.two || o.bias || rank[i] == -INFINITY ? rank[i] : score[i];
        }
        __builtin_amdgcn_wave_barrier();
        double best = -INFINITY, second = -INFINITY;
        if (lane < o.groups)
            for (int i = 0; i < per; i++) {
                const double r = mine[lane * per + i];
                if (r > best) second = best, best = r;
                else if (r > second) second = r;
            }
        double of_group = o.two && second > -INFINITY ? best + second : best;
        uint64_t kept = 0;
        for (int j = 0; j < o.top_groups; j++) {
            double r = of_group;
            int g = lane;
            wave_best(r, g);
            if (r == -INFINITY) break;
            kept |= 1ull << g;
            if (lane == g) of_group = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < EPL; i++) {
            const int e = lane + 64 * i;
            if (e < o.experts && !(kept >> (e / per) & 1)) rank[i] = -INFINITY;
        }
    }
    int id = -1;           // the lane's choice, and its score
    double chosen = 0.0, total = 0.0;
    for (int j = 0; j < o.choices; j++) {
        double r = -INFINITY, its = 0.0;
        int e = INT32_MAX;
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (rank[i] > r) r = rank[i], e = lane + 64 * i;
        wave_best(r, e);
        if (r == -INFINITY) break;
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (e == lane + 64 * i) {
                its = score[i];
                rank[i] = -INFINITY;
            }
        its = __shfl(its, e % 64);
        total += its;
        if (lane == j) id = e, chosen = its;
    }
    if (lane < o.choices) {
        double w = o.scale * chosen;
        if (o.renormalise) w = total > 0.0 ? w / total : 0.0;
        ids[t * o.choices + lane] = id;
        weights[t * o.choices + lane] = spoilt ? NAN : id < 0 ? 0.f : (float)w;
    }
}

// With g the gradient of the weights, c the scale, s the scores, S their sum over the chosen ones and q_j = s_j / S:
//   softmax, renormalised    dx_i = c q_i (g_i - sum_j g_j q_j) for the chosen, else 0
//   softmax                  dx_i = c s_i ([i chosen] g_i - sum_j g_j s_j)
//   sigmoid, renormalised    dx_i = c q_i (1 - s_i) (g_i - sum_j g_j q_j) for the chosen, else 0
//   sigmoid                  dx_i = c s_i (1 - s_i) g_i for the chosen, else 0
template <typename T, int EPL>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(const T *logits, int64_t stride, int64_t tokens, Options o, const int *ids, const float *grad,
                                                                  T *out) {
    const int lane = threadIdx.x % 64;
    const int64_t t = (int64_t)blockIdx.x * kTokensAtOnce + threadIdx.x / 64;
    if (t >= tokens) return;
    double x[EPL], score[EPL], g[EPL];
    bool spoilt, chosen[EPL];
    scores_of<T, EPL>(logits + t * stride, o, lane, x, score, spoilt);
#pragma unroll
    for (int i = 0; i < EPL; i++) chosen[i] = false, g[i] = 0.0;
    for (int j = 0; j < o.choices; j++) {
        const int e = ids[t * o.choices + j];
        const double its = grad[t * o.choices + j];
#pragma unroll
        for (int i = 0; i < EPL; i++)
            if (e == lane + 64 * i) chosen[i] = true, g[i] = its;
    }
    double sum = 0.0, total = 1.0;
    if (o.renormalise) {
        total = 0.0;
#pragma unroll
        for (int i = 0; i < EPL; i++) total += chosen[i] ? score[i] : 0.0;
        total = wave_sum(total);
    }
    if (o.renormalise || !o.sigmoid) {
#pragma unroll
        for (int i = 0; i < EPL; i++) sum += chosen[i] ? g[i] * score[i] : 0.0;
        sum = wave_sum(sum);
        if (total > 0.0) sum /= total;
    }
#pragma unroll
    for (int i = 0; i < EPL; i++) {
        const int e = lane + 64 * i;
        double d = 0.0;
        if (total > 0.0 && (chosen[i] || (!o.renormalise && !o.sigmoid))) d = o.scale * (score[i] / total) * (g[i] - sum) * (o.sigmoid ? 1.0 - score[i] : 1.0);
        if (e < o.experts) out[t * o.experts + e] = from_float<T>(spoilt ? NAN : (float)d);
    }
}

template <typename T, int EPL>
void route(const void *logits, int64_t stride, int64_t tokens, const Options &o, int *ids, float *weights, hipStream_t s) {
    const size_t room = o.groups > 1 ? sizeof(double) * kTokensAtOnce * o.experts : 0;
    route_kernel<T, EPL><<<(unsigned)((tokens + kTokensAtOnce - 1) / kTokensAtOnce), kThreads, room, s>>>((const T *)logits, stride, tokens, o, ids, weights);
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
    return {o->experts, o->choices, o->groups, o->top_groups, o->sigmoid != 0, o->group_two != 0, o->renormalise != 0, o->scale, o->bias};
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
