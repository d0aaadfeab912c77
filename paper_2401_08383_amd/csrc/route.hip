// moe_route, moe_route_backward: ids and weights of a token's experts from its logits, and the gradient of the logits.
//
// A token belongs to L lanes of a wavefront, V consecutive experts to a lane, so that a lower lane and a lower register hold lower ids.
// Slot j of the choice is kept by lane j of the token.
#include <math.h>

#include <type_traits>

#include "product.hpp"

namespace exf {

struct RouteCall {
    const void* logits;
    const float* bias;  // [E] or null
    int32_t* idx;
    float* w;
    float* scores;      // [T,E] or null
    int64_t T;
    int E, k, groups, top_groups, group_best, renormalize;
    float scale;
};

struct RouteGradient {
    const void* logits;
    const int32_t* idx;
    const float* dw;
    const float* dscores;  // a row of E every `dscores_stride`, or null
    int64_t dscores_stride;
    void* dlogits;
    int64_t T;
    int E, k, renormalize;
    float scale;
};

constexpr int kRouteThreads = 256;

// Reductions over the L lanes of a token, in every lane.
template <int L, class F>
__device__ __forceinline__ float over_token(float v, F f)
{
    float a, b;
    if constexpr (L >= 32) butterfly<16>(v, a, b), v = f(a, b);
    butterfly<8>(v, a, b), v = f(a, b);
    butterfly<4>(v, a, b), v = f(a, b);
    butterfly<2>(v, a, b), v = f(a, b);
    butterfly<1>(v, a, b), v = f(a, b);
    return v;
}
template <int L>
__device__ __forceinline__ float token_max(float v) { return over_token<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ __forceinline__ float token_sum(float v) { return over_token<L>(v, [](float a, float b) { return a + b; }); }
template <int L>
__device__ __forceinline__ double token_sum64(double v)
{
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// V logits of experts first .. first + V - 1 of a row, -inf past the last one.
template <bool BF16>
__device__ __forceinline__ float load_logit(const void* row, int e)
{
    if constexpr (BF16) return bf16_to_f32(static_cast<const bf16_t*>(row)[e]);
    else return static_cast<const float*>(row)[e];
}
template <bool BF16>
__device__ __forceinline__ const void* row_at(const void* p, int64_t i) { return static_cast<const uint8_t*>(p) + i * (BF16 ? 2 : 4); }
template <int V, bool BF16>
__device__ __forceinline__ void load_logits(const void* row, int first, int E, float (&l)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = first + v < E ? load_logit<BF16>(row, first + v) : -INFINITY;
}

// Weights of the chosen experts, lane j of the token with logit l of its own (live: there is one); `most` and `sum`: the largest logit of the
// token and the sum of exp(l - most).
//   Renormalised scores are u_j / sum u with any u proportional to the scores: exp(l - the largest chosen l) for the softmax, and for the sigmoid
// 1 / (1 + exp(-l)), or where no chosen logit is positive e^-c / (1 + exp(-l)) = exp(l - c) / (1 + exp(l)) with c the largest of them: no sum underflows.
template <int L, bool SIGMOID>
__device__ __forceinline__ float chosen_share(float l, bool live)
{
    const float top = token_max<L>(live ? l : -INFINITY);
    float u;
    if constexpr (SIGMOID) u = l > 0.0f ? 1.0f / (1.0f + expf(-l)) : expf(l - fminf(top, 0.0f)) / (1.0f + expf(l));
    else u = expf(l - top);
    if (!live) u = 0.0f;
    const float all = token_sum<L>(u);
    return live ? u / all : 0.0f;
}
__device__ __forceinline__ float sigmoid(float l)
{
    const float t = expf(-fabsf(l));
    return (l >= 0.0f ? 1.0f : t) / (1.0f + t);
}
__device__ __forceinline__ double sigmoid64(double l)
{
    const double t = exp(-fabs(l));
    return (l >= 0.0 ? 1.0 : t) / (1.0 + t);
}

// Scans of a lane's keys keep the earlier of equals; of lanes, the lower one.
template <int L>
__device__ __forceinline__ void best_over_token(double& key, int& at)
{
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) {
        const double k2 = __shfl_xor(key, off, kWave);
        const int a2 = __shfl_xor(at, off, kWave);
        const bool second = k2 > key || (k2 == key && a2 < at);
        key = second ? k2 : key;
        at = second ? a2 : at;
    }
}

template <int V, int L, bool BF16, bool SIGMOID>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(const RouteCall p)
{
    const int lane = lane_id(), in = lane % L;
    constexpr int kTokens = kRouteThreads / L;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens; t0 < p.T; t0 += static_cast<int64_t>(gridDim.x) * kTokens) {
    const int64_t t = t0 + threadIdx.x / L;
    const bool there = t < p.T;
    const int64_t row = min(t, p.T - 1);
    const void* at = row_at<BF16>(p.logits, row * p.E);
    const int first = in * V;
    float l[V];
    load_logits<V, BF16>(at, first, p.E, l);
    float most = -INFINITY;
    bool broken = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        most = fmaxf(most, l[v]);  // (ignores a NaN)
        broken |= l[v] != l[v];
    }
    most = token_max<L>(most);
    broken = token_max<L>(broken ? 1.0f : 0.0f) > 0.0f || (!SIGMOID && most == INFINITY);
    const float base = most == -INFINITY ? 0.0f : most;
    float sum = 0.0f;
    if constexpr (!SIGMOID) {
#pragma unroll
        for (int v = 0; v < V; ++v) sum += expf(l[v] - base);
        sum = token_sum<L>(sum);
    }
    if (p.scores != nullptr && there) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (first + v < p.E) p.scores[row * p.E + first + v] = SIGMOID ? sigmoid(l[v]) : (most == -INFINITY ? 0.0f : expf(l[v] - base) / sum);
    }

    // keys in 64 bits
    double key[V];
    const bool wide = p.bias != nullptr || (p.groups > 1 && p.group_best == 2);
    double sum64 = 0.0;
    if (wide && !SIGMOID) {
#pragma unroll
        for (int v = 0; v < V; ++v) sum64 += l[v] > -INFINITY ? exp(static_cast<double>(l[v]) - base) : 0.0;
        sum64 = token_sum64<L>(sum64);
    }
    auto score64 = [&](float v) -> double { return SIGMOID ? sigmoid64(v) : exp(static_cast<double>(v) - base) / sum64; };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        key[v] = l[v];
        if (p.bias != nullptr) key[v] = score64(l[v]) + p.bias[min(first + v, p.E - 1)];
        if (!(l[v] > -INFINITY) || !(key[v] > -INFINITY)) key[v] = -INFINITY;  // (also a NaN)
    }
    if (p.groups > 1) {
        const int size = p.E / p.groups;
        unsigned long long stay = ~0ull;
        double mine[kWave / L];  // values of groups in, in + L, ...
#pragma unroll
        for (int q = 0; q < kWave / L; ++q) mine[q] = -INFINITY;
        for (int g = 0; g < p.groups; ++g) {
            double a = -INFINITY, b = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const bool member = first + v >= g * size && first + v < (g + 1) * size && key[v] > -INFINITY;
                const double s = member ? (p.bias == nullptr && p.group_best == 2 ? score64(l[v]) : key[v]) : -INFINITY;
                b = fmax(b, fmin(a, s));
                a = fmax(a, s);
            }
#pragma unroll
            for (int off = L / 2; off > 0; off >>= 1) {
                const double a2 = __shfl_xor(a, off, kWave), b2 = __shfl_xor(b, off, kWave);
                b = fmax(fmax(b, b2), fmin(a, a2));
                a = fmax(a, a2);
            }
            if (p.group_best == 2 && b > -INFINITY) a += b;
#pragma unroll
            for (int q = 0; q < kWave / L; ++q)
                if (g == in + q * L) mine[q] = a;
        }
        stay = 0ull;
        for (int j = 0; j < p.top_groups; ++j) {
            double a = -INFINITY;
            int g = kWave;
#pragma unroll
            for (int q = 0; q < kWave / L; ++q)
                if (mine[q] > a) a = mine[q], g = in + q * L;
            best_over_token<L>(a, g);
            if (g < kWave) stay |= 1ull << g;
#pragma unroll
            for (int q = 0; q < kWave / L; ++q)
                if (g == in + q * L) mine[q] = -INFINITY;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (((stay >> min((first + v) / size, kWave - 1)) & 1ull) == 0ull) key[v] = -INFINITY;
    }

    int chosen = -1;
    for (int j = 0; j < p.k; ++j) {
        double a = -INFINITY;
        int e = 1 << 20;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (key[v] > a) a = key[v], e = first + v;
        best_over_token<L>(a, e);
        if (in == j && a > -INFINITY) chosen = e;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (first + v == e) key[v] = -INFINITY;
    }
    const bool live = chosen >= 0;
    const float mine = live ? load_logit<BF16>(at, chosen) : -INFINITY;
    float w;
    if (p.renormalize && p.k > 1) w = chosen_share<L, SIGMOID>(mine, live);
    else if (!live) w = 0.0f;
    else w = SIGMOID ? sigmoid(mine) : expf(mine - base) / sum;
    if (there && in < p.k) {
        p.idx[row * p.k + in] = chosen;
        p.w[row * p.k + in] = broken ? NAN : p.scale * w;
    }
    }
}

// dw -> dlogits (g = dw, u = a chosen expert's share of the chosen scores, w = scale u or scale s):
//   renormalised: the chosen experts' w_j (g_j - sum_i g_i u_i), times 1 - s_j for the sigmoid
//   sigmoid:      scale g_j s_j (1 - s_j)
//   softmax:      scale g_j p_j at the chosen ones, less p_e sum_j scale g_j p_j at all
// and of the scores' own gradient d: d_e s_e (1 - s_e), or p_e (d_e - sum d p).
template <int V, int L, bool BF16, bool SIGMOID>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(const RouteGradient p)
{
    const int lane = lane_id(), in = lane % L;
    constexpr int kTokens = kRouteThreads / L;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens; t0 < p.T; t0 += static_cast<int64_t>(gridDim.x) * kTokens) {
    const int64_t t = t0 + threadIdx.x / L;
    const bool there = t < p.T;
    const int64_t row = min(t, p.T - 1);
    const void* at = row_at<BF16>(p.logits, row * p.E);
    const int first = in * V;
    const bool renormalize = p.renormalize && p.k > 1;
    const int e = in < p.k ? p.idx[row * p.k + in] : -1;
    const bool live = e >= 0 && e < p.E;
    const float mine = live ? load_logit<BF16>(at, e) : -INFINITY, g = live ? p.dw[row * p.k + in] : 0.0f;

    float out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = 0.0f;
    float most = 0.0f, sum = 1.0f, less = 0.0f, change = 0.0f;
    float l[V], d[V];
    const bool all = p.dscores != nullptr || (!SIGMOID && !renormalize);
    if (all) {
        load_logits<V, BF16>(at, first, p.E, l);
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = p.dscores != nullptr && first + v < p.E ? p.dscores[row * p.dscores_stride + first + v] : 0.0f;
        if constexpr (!SIGMOID) {
            most = l[0];
#pragma unroll
            for (int v = 1; v < V; ++v) most = fmaxf(most, l[v]);
            most = token_max<L>(most);
            if (most == -INFINITY) most = 0.0f;
            sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[v] = expf(l[v] - most);
                sum += l[v];
            }
            sum = token_sum<L>(sum);
            if (sum == 0.0f) sum = 1.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[v] /= sum;
                less += l[v] != 0.0f ? l[v] * d[v] : 0.0f;  // (a score of a masked expert, whatever its gradient)
            }
            less = token_sum<L>(less);
        }
    }
    if (renormalize) {
        const float u = chosen_share<L, SIGMOID>(mine, live && mine > -INFINITY);
        const float mean = token_sum<L>(g * u);
        change = p.scale * u * (g - mean);
        if constexpr (SIGMOID) change *= sigmoid(-mine);
    } else if constexpr (SIGMOID) {
        change = p.scale * g * sigmoid(mine) * sigmoid(-mine);
    } else {
        change = p.scale * g * (expf(mine - most) / sum);
        less += token_sum<L>(change);
    }
    if (!live) change = 0.0f;
    if (all) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float slope = SIGMOID ? sigmoid(l[v]) * sigmoid(-l[v]) : l[v];
            out[v] = slope != 0.0f ? slope * (SIGMOID ? d[v] : d[v] - less) : 0.0f;
        }
    }
    for (int j = 0; j < p.k; ++j) {
        const int ej = __shfl(live ? e : -1, (lane & ~(L - 1)) + j, kWave);
        const float cj = __shfl(change, (lane & ~(L - 1)) + j, kWave);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (first + v == ej) out[v] += cj;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (there && first + v < p.E) {
            if constexpr (BF16) static_cast<bf16_t*>(p.dlogits)[row * p.E + first + v] = f32_to_bf16(out[v]);
            else static_cast<float*>(p.dlogits)[row * p.E + first + v] = out[v];
        }
    }
}

// Calls run(V, L, type, score) with the instance for E experts.
template <class F>
static void pick_route(int E, int dt, int score, F run)
{
    auto with = [&](auto v, auto l) {
        const std::true_type yes;
        const std::false_type no;
        if (dt == EXF_BF16) score == EXF_SCORE_SIGMOID ? run(v, l, yes, yes) : run(v, l, yes, no);
        else score == EXF_SCORE_SIGMOID ? run(v, l, no, yes) : run(v, l, no, no);
    };
    const std::integral_constant<int, 16> l16;
    const std::integral_constant<int, 32> l32;
    if (E <= 64) with(std::integral_constant<int, 4>(), l16);
    else if (E <= 128) with(std::integral_constant<int, 8>(), l16);
    else if (E <= 256) with(std::integral_constant<int, 16>(), l16);
    else with(std::integral_constant<int, 16>(), l32);
}

static unsigned route_grid(int64_t T, int tokens)
{
    const int64_t blocks = (T + tokens - 1) / tokens;
    return static_cast<unsigned>(blocks < (1 << 20) ? blocks : 1 << 20);
}

static int check_route(const char* fn, int64_t T, int E, int k, int score, float scale, int dt)
{
    if (dt != EXF_F32 && dt != EXF_BF16) return fail(EXF_ERR_BAD_DTYPE, "%s: dt = %d", fn, dt);
    if (T < 0) return fail(EXF_ERR_BAD_SHAPE, "%s: T = %lld < 0", fn, static_cast<long long>(T));
    if (E < 1 || E > EXF_MAX_ROUTE_EXPERTS) return fail(EXF_ERR_BAD_SHAPE, "%s: E = %d outside [1,%d]", fn, E, EXF_MAX_ROUTE_EXPERTS);
    if (k < 1 || k > EXF_MAX_ROUTE_TOPK || k > E) return fail(EXF_ERR_BAD_SHAPE, "%s: k = %d outside [1,min(E,%d)]", fn, k, EXF_MAX_ROUTE_TOPK);
    if (T >= (1ll << 31) / k) return fail(EXF_ERR_BAD_SHAPE, "%s: T*k must be below 2^31", fn);
    if (score != EXF_SCORE_SOFTMAX && score != EXF_SCORE_SIGMOID) return fail(EXF_ERR_BAD_SHAPE, "%s: score = %d", fn, score);
    if (!isfinite(scale)) return fail(EXF_ERR_BAD_SHAPE, "%s: scale must be finite", fn);
    return EXF_OK;
}

}  // namespace exf

extern "C" int moe_route(const void* logits, const float* bias, int64_t T, int E, int k, int score, int groups, int top_groups, int group_best,
                         int renormalize, float scale, int dt, int32_t* topk_idx, float* topk_w, float* scores_out, void* stream)
{
    using namespace exf;
    const char* fn = "moe_route";
    if (int rc = check_route(fn, T, E, k, score, scale, dt)) return rc;
    if (groups < 1 || groups > EXF_MAX_ROUTE_GROUPS || E % groups != 0)
        return fail(EXF_ERR_BAD_SHAPE, "%s: groups = %d must divide E = %d and not exceed %d", fn, groups, E, EXF_MAX_ROUTE_GROUPS);
    if (top_groups < 1 || top_groups > groups) return fail(EXF_ERR_BAD_SHAPE, "%s: top_groups = %d outside [1,%d]", fn, top_groups, groups);
    if (group_best != 1 && group_best != 2) return fail(EXF_ERR_BAD_SHAPE, "%s: group_best = %d is neither 1 nor 2", fn, group_best);
    if (k > top_groups * (E / groups)) return fail(EXF_ERR_BAD_SHAPE, "%s: k = %d of %d groups of %d experts", fn, k, top_groups, E / groups);
    if (T == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, logits);
    EXF_CHECK_PTR(fn, topk_idx);
    EXF_CHECK_PTR(fn, topk_w);
    EXF_CHECK_ALIGNED(fn, logits);
    if (scores_out != nullptr) EXF_CHECK_ALIGNED(fn, scores_out);
    const size_t n = static_cast<size_t>(T) * E, in = n * (dt == EXF_BF16 ? 2 : 4), slots = static_cast<size_t>(T) * k * 4, experts = static_cast<size_t>(E) * 4;
    const struct {
        const void* at;
        size_t bytes;
    } out[] = {{topk_idx, slots}, {topk_w, slots}, {scores_out, n * 4}};
    for (int i = 0; i < 3; ++i) {
        if (overlap(out[i].at, out[i].bytes, logits, in) || overlap(out[i].at, out[i].bytes, bias, experts))
            return fail(EXF_ERR_BAD_SHAPE, "%s: results must not overlap an input", fn);
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return fail(EXF_ERR_BAD_SHAPE, "%s: results must not overlap", fn);
    }
    const RouteCall p{logits, bias, topk_idx, topk_w, scores_out, T, E, k, groups == top_groups ? 1 : groups, top_groups, group_best, renormalize, scale};
    pick_route(E, dt, score, [&](auto v, auto l, auto bf16, auto sigmoid) {
        constexpr int kTokens = kRouteThreads / decltype(l)::value;
        hipLaunchKernelGGL((route_kernel<decltype(v)::value, decltype(l)::value, decltype(bf16)::value, decltype(sigmoid)::value>),
                           dim3(route_grid(T, kTokens)), dim3(kRouteThreads), 0, static_cast<hipStream_t>(stream), p);
    });
    return check_launch(fn);
}

extern "C" int moe_route_backward(const float* dtopk_w, const void* logits, const int32_t* topk_idx, const float* dscores, int64_t dscores_stride, int64_t T,
                                  int E, int k, int score, int renormalize, float scale, int dt, void* dlogits, void* stream)
{
    using namespace exf;
    const char* fn = "moe_route_backward";
    if (int rc = check_route(fn, T, E, k, score, scale, dt)) return rc;
    if (dscores != nullptr && dscores_stride != 0 && dscores_stride != E)
        return fail(EXF_ERR_BAD_SHAPE, "%s: dscores_stride = %lld is neither 0 nor E", fn, static_cast<long long>(dscores_stride));
    if (T == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, dtopk_w);
    EXF_CHECK_PTR(fn, logits);
    EXF_CHECK_PTR(fn, topk_idx);
    EXF_CHECK_PTR(fn, dlogits);
    EXF_CHECK_ALIGNED(fn, logits);
    EXF_CHECK_ALIGNED(fn, dlogits);
    if (dscores != nullptr) EXF_CHECK_ALIGNED(fn, dscores);
    const size_t n = static_cast<size_t>(T) * E, el = dt == EXF_BF16 ? 2 : 4, slots = static_cast<size_t>(T) * k * 4;
    if (overlap(dlogits, n * el, logits, n * el) || overlap(dlogits, n * el, dtopk_w, slots) || overlap(dlogits, n * el, topk_idx, slots) ||
        overlap(dlogits, n * el, dscores, dscores_stride == 0 ? static_cast<size_t>(E) * 4 : n * 4))
        return fail(EXF_ERR_BAD_SHAPE, "%s: the result must not overlap an input", fn);
    const RouteGradient p{logits, topk_idx, dtopk_w, dscores, dscores_stride, dlogits, T, E, k, renormalize, scale};
    pick_route(E, dt, score, [&](auto v, auto l, auto bf16, auto sigmoid) {
        constexpr int kTokens = kRouteThreads / decltype(l)::value;
        hipLaunchKernelGGL((route_backward_kernel<decltype(v)::value, decltype(l)::value, decltype(bf16)::value, decltype(sigmoid)::value>),
                           dim3(route_grid(T, kTokens)), dim3(kRouteThreads), 0, static_cast<hipStream_t>(stream), p);
    });
    return check_launch(fn);
}
