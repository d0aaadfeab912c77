// moe_route, moe_route_backward: ids and weights of a token's experts from its logits, and the gradient of the logits.
//
// A token belongs to L lanes of a wavefront, V consecutive experts to a lane, so that a lower lane and a lower register hold lower ids.
// Slot j of the choice is kept by lane j of the token.
//   What bounds it: reading takes 6 us of the 25.4 of 32768 tokens, 8 of 256 experts in 8 groups, sigmoid, bias, fp32 (calls in a graph); vector instructions the rest, 1160 a
// wavefront of four tokens (350 of them for the groups).  Without groups 18.4; without a bias sigmoid 13.8, softmax of fp32 logits 15.7 and of bf16 ones 13.6, renormalised, which needs no
// sum over all experts, 11.6; keys of 64 bits throughout 98.  Registers for a fifth wavefront a SIMD (96 of 119, some spilled) gain nothing, 28.  One token 3.2 (2.7 by itself), in groups
// 5.4: loads that follow one another and nine turns of a maximum over lanes.
//   The gradient of 32768 x 256 fp32 logits: with that of the scores 16 to 18 us for 69 MB, 4.1 TB/s; without it 11.3 where only the chosen ones are read (33.5 MB are written), 16.8 of
// softmax weights that are not renormalised; of bf16 logits 9.0 and 13.3.
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

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* row, int e)
{
    if constexpr (BF16) return bf16_to_f32(static_cast<const bf16_t*>(row)[e]);
    else return static_cast<const float*>(row)[e];
}
// A logit's place in the order of all bf16 numbers, from 1 on; 0 for -inf and NaN.
__device__ __forceinline__ uint32_t ordered(float l)
{
    const uint32_t u = __float_as_uint(l + 0.0f) >> 16;  // (-0 is 0)
    return l > -INFINITY ? ((u & 0x8000u) != 0u ? 0xffffu - u : u + 0x8000u) + 1u : 0u;
}
template <bool BF16>
__device__ __forceinline__ const void* row_at(const void* p, int64_t i) { return static_cast<const uint8_t*>(p) + i * (BF16 ? 2 : 4); }
// A lane's experts are first + place(0), first + place(1), ..: pieces of four, P apart, with those of the other lanes between them, so that neighbouring lanes
// load what lies together: 16 accesses to the L1 instead of 64 (gradient of 32768 x 256 fp32 logits with that of the scores: 22.9 us with V next to each other, 16.4 when this was done).
template <int P>
__host__ __device__ constexpr int place(int v) { return v / 4 * P + v % 4; }

// The lane's V values of a row, `none` past the last one; four at a time where rows are a multiple of that.
template <int V, int P, bool BF16>
__device__ __forceinline__ void load_row(const void* row, int first, int E, float none, float (&l)[V], bool aligned = true)
{
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = none;
    if (E % 4 == 0 && aligned) {
#pragma unroll
        for (int v = 0; v < V; v += 4)
            if (first + place<P>(v) < E) {
                if constexpr (BF16) {
                    const uint2 t = *reinterpret_cast<const uint2*>(static_cast<const bf16_t*>(row) + first + place<P>(v));
                    l[v] = __uint_as_float(t.x << 16), l[v + 1] = __uint_as_float(t.x & 0xffff0000u);
                    l[v + 2] = __uint_as_float(t.y << 16), l[v + 3] = __uint_as_float(t.y & 0xffff0000u);
                } else {
                    const float4 t = *reinterpret_cast<const float4*>(static_cast<const float*>(row) + first + place<P>(v));
                    l[v] = t.x, l[v + 1] = t.y, l[v + 2] = t.z, l[v + 3] = t.w;
                }
            }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float x = load_logit<BF16>(row, min(first + place<P>(v), E - 1));
            l[v] = first + place<P>(v) < E ? x : none;
        }
    }
}
template <int V, int P, bool BF16>
__device__ __forceinline__ void store_row(void* row, int first, int E, const float (&l)[V])
{
    if (E % 4 == 0) {
#pragma unroll
        for (int v = 0; v < V; v += 4)
            if (first + place<P>(v) < E) {
                if constexpr (BF16) *reinterpret_cast<uint2*>(static_cast<bf16_t*>(row) + first + place<P>(v)) = make_uint2(pack_bf16x2(l[v], l[v + 1]), pack_bf16x2(l[v + 2], l[v + 3]));
                else *reinterpret_cast<float4*>(static_cast<float*>(row) + first + place<P>(v)) = make_float4(l[v], l[v + 1], l[v + 2], l[v + 3]);
            }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (first + place<P>(v) < E) {
                if constexpr (BF16) static_cast<bf16_t*>(row)[first + place<P>(v)] = f32_to_bf16(l[v]);
                else static_cast<float*>(row)[first + place<P>(v)] = l[v];
            }
    }
}

// exp(x) for x <= 0 (0 below -200), to less than two units: what the argument loses on its way to base 2 is put back by a second part of log2 e (the two-part reduction of
// Cody and Waite), and results below the normal range are kept (the instruction flushes them).
__device__ __forceinline__ float exp_below(float x)
{
    x = x < -200.0f ? -200.0f : x;
    const float whole = rintf(x * 1.442695041f);
    return ldexpf(__builtin_amdgcn_exp2f(fmaf(x, 1.925963033e-8f, fmaf(x, 1.442695041f, -whole))), static_cast<int>(whole));
}
// a / b for b in [1/2, 16] and a in [0, b], to a unit: by a reciprocal, its remainder put back (as Markstein does).
__device__ __forceinline__ float quotient(float a, float b)
{
    const float r = __builtin_amdgcn_rcpf(b), q = a * r;
    return fmaf(fmaf(-b, q, a), r, q);
}
__device__ __forceinline__ float sigmoid(float l)
{
    const float t = exp_below(-fabsf(l));
    return quotient(l >= 0.0f ? 1.0f : t, 1.0f + t);
}
// s (1 - s) of s = sigmoid(l), also where s is next to 1.
__device__ __forceinline__ float sigmoid_slope(float l)
{
    const float t = exp_below(-fabsf(l)), q = quotient(1.0f, 1.0f + t);
    return t * q * q;
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
    if constexpr (SIGMOID) u = quotient(l > 0.0f ? 1.0f : exp_below(l - fminf(top, 0.0f)), 1.0f + exp_below(-fabsf(l)));
    else u = exp_below(l - top);
    if (!live) u = 0.0f;
    const float all = token_sum<L>(u);  // (from 1/2, that of the largest, to 16)
    return live ? quotient(u, all) : 0.0f;
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

// Ids by keys in 64 bits, in the order of the definition; slot j in lane j.  `keys`: the lane's logits, kWave apart.  In LDS and in loops:
// wavefronts that need none of it would have to leave room for its registers (245 instead of 90 with 16 experts a lane, two wavefronts a SIMD: 32768 tokens of 256
// experts in groups 50 us).
template <int V, int P, int L, bool SIGMOID, bool SCORES, bool GROUPS>
__device__ __forceinline__ int choose_exactly(const RouteCall& p, double* keys, int first, int in, float base)
{
    const bool by_score = SCORES && p.bias == nullptr;  // (of groups)
    double sum64 = 0.0;
    if constexpr (SCORES && !SIGMOID) {
#pragma unroll 1
        for (int v = 0; v < V; ++v) {
            const double x = keys[v * kWave];
            sum64 += x > -INFINITY ? exp(x - base) : 0.0;
        }
        sum64 = token_sum64<L>(sum64);
    }
    auto score64 = [&](double x) -> double { return SIGMOID ? sigmoid64(x) : exp(x - base) / sum64; };
#pragma unroll 1
    for (int v = 0; v < V; ++v) {
        const double x = keys[v * kWave];
        double key = x;
        if (SCORES && p.bias != nullptr) key = score64(x) + p.bias[min(first + place<P>(v), p.E - 1)];
        keys[v * kWave] = x > -INFINITY && key > -INFINITY ? key : -INFINITY;  // (out: also a NaN)
    }
    unsigned long long stay = ~0ull;
    const int size = p.E / p.groups;
    if constexpr (GROUPS) {
        double mine[kWave / L];  // values of groups in, in + L, ...
#pragma unroll
        for (int q = 0; q < kWave / L; ++q) mine[q] = -INFINITY;
#pragma unroll 1
        for (int g = 0; g < p.groups; ++g) {
            double a = -INFINITY, b = -INFINITY;
#pragma unroll 1
            for (int v = 0; v < V; ++v) {
                const int e = first + place<P>(v);
                double s = e >= g * size && e < (g + 1) * size ? keys[v * kWave] : -INFINITY;
                if (by_score && s > -INFINITY) s = score64(s);
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
#pragma unroll 1
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
    }
    int chosen = -1;
#pragma unroll 1
    for (int j = 0; j < p.k; ++j) {
        double a = -INFINITY;
        int e = 1 << 20;
#pragma unroll 1
        for (int v = 0; v < V; ++v) {
            const double key = keys[v * kWave];
            if (key > a && (!GROUPS || ((stay >> min((first + place<P>(v)) / size, kWave - 1)) & 1ull) != 0ull)) a = key, e = first + place<P>(v);
        }
        best_over_token<L>(a, e);
        if (in == j && a > -INFINITY) chosen = e;
        const int off = e - first, slot = off / P * 4 + off % P;
        if (off >= 0 && off % P < 4 && slot < V) keys[slot * kWave] = -INFINITY;
    }
    return chosen;
}

// ---- the same by whole numbers of 32 bits, where they are sure of the order
// A key's place between the least and the largest of its token, in 2^22 steps, is its class; the number (class, 511 - id) is unique, the largest one is found
// with one instruction a step, and equals go to the lowest id.  Where the classes of two experts that follow one another - the last chosen one and the next
// included - are further apart than the classes' own error, so are the keys; otherwise the wavefront begins again in 64 bits.
//   bf16 logits without a bias: a class is the logit itself, and always sure.
constexpr int kIdBits = 9;
static_assert(EXF_MAX_ROUTE_EXPERTS <= 1 << kIdBits, "an id has its bits");
constexpr float kClasses = 4194304.0f;  // 2^22

template <int L>
__device__ __forceinline__ uint32_t token_max_u32(uint32_t v)
{
    uint32_t a, b;
    if constexpr (L >= 32) butterfly<16>(v, a, b), v = max(a, b);
    butterfly<8>(v, a, b), v = max(a, b);
    butterfly<4>(v, a, b), v = max(a, b);
    butterfly<2>(v, a, b), v = max(a, b);
    butterfly<1>(v, a, b), v = max(a, b);
    return v;
}

// Sorted, the largest first (odd-even merge sort).
template <int V>
__device__ __forceinline__ void sort_keys(uint32_t (&s)[V])
{
#pragma unroll
    for (int p = 1; p < V; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < V; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < V && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const uint32_t a = s[i + j], b = s[i + j + k];
                        s[i + j] = max(a, b), s[i + j + k] = min(a, b);
                    }
}

// The keys of lanes i and i ^ OFF, the same pair in both of them; lanes that differ in lower bits agree already.
template <int OFF>
__device__ __forceinline__ uint32_t other_lane(uint32_t v)
{
    if constexpr (OFF == 1) return __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);        // quad_perm 1,0,3,2
    else if constexpr (OFF == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);   // quad_perm 2,3,0,1
    else if constexpr (OFF == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);  // row_half_mirror
    else if constexpr (OFF == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);  // row_mirror
    else return static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), OFF, kWave));
}
template <int OFF>
__device__ __forceinline__ void best_two(uint32_t& a, uint32_t& b)
{
    const uint32_t a2 = other_lane<OFF>(a), b2 = other_lane<OFF>(b);
    b = max(max(b, b2), min(a, a2));
    a = max(a, a2);
}

// Largest of the finite values above the lowest that stand for masks, the least of them, and 2^22 steps between them.
//   Masks are -inf and what is not above -1e30.  fp32 logits without a bias that are masked by a number nearer to zero leave few steps for the others: with -1e9 none, and rows
// with more of them than the token has lanes are put in order by keys in 64 bits, 50 us where -inf takes 15.7 (32768 x 256, 30 % masked); with -1e4 21.  (Scores and bf16 logits do not mind.)
struct Classes {
    float most, step;
};
template <int V, int L>
__device__ __forceinline__ Classes classes_of(const float (&key)[V])
{
    float most = -INFINITY, least = INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        most = fmaxf(most, key[v]);
        least = fminf(least, key[v] > -1e30f ? key[v] : INFINITY);
    }
    most = token_max<L>(most);
    least = -token_max<L>(-least);
    const float range = most - least;
    return {most, range > 0.0f && range < 1e30f ? (kClasses - 2.0f) * __builtin_amdgcn_rcpf(range) : 0.0f};
}
// 0: out; 1: at the least, or below; otherwise in order, to within one.  (What is out may have widened the range: classes are coarser then, and in order.)
__device__ __forceinline__ uint32_t class_of(float key, Classes c, float logit)
{
    const float at = fmaf(key - c.most, c.step, kClasses);
    return logit > -INFINITY && key > -INFINITY ? static_cast<uint32_t>(fmaxf(at, 1.0f)) : 0u;
}

// LDS of a wavefront is written and read in order; this keeps the compiler from moving either.
__device__ __forceinline__ void lds_in_order()
{
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Where a group's lanes are, if not those that hold its experts: `parts` lanes a group, each with a share of its experts (at most L groups).
template <int L>
struct GroupParts {
    int parts, mine, begin, end;  // my group; its experts that are mine
    __device__ GroupParts(int E, int groups, int in)
    {
        const int size = E / groups;
        parts = L;
        while (parts * groups > L) parts >>= 1;
        mine = in / parts;
        const int share = (size + parts - 1) / parts, part = in % parts;
        begin = mine * size + min(part * share, size);
        end = mine < groups ? mine * size + min((part + 1) * share, size) : begin;
    }
};

// The logits of the token's lanes as they lie in a row, at `mine`, for all of them.
template <int V, int P, int L>
__device__ __forceinline__ void share_logits(const float (&l)[V], float* token, int first)
{
    lds_in_order();
#pragma unroll
    for (int v = 0; v < V; ++v) token[first + place<P>(v)] = l[v];
    lds_in_order();
}

// Score and key of a logit in 64 bits; -inf: out.
template <int V, int P, int L, bool SIGMOID, bool SCORES>
struct ExactKeys {
    const float* bias;
    float base;
    double sum;
    __device__ ExactKeys(const float* bias, const float* token, int first, float base) : bias(bias), base(base), sum(0.0)
    {
        if constexpr (SCORES && !SIGMOID) {
#pragma unroll 1
            for (int v = 0; v < V; ++v) {
                const float x = token[first + place<P>(v)];
                sum += x > -INFINITY ? exp(static_cast<double>(x) - base) : 0.0;
            }
            sum = token_sum64<L>(sum);
        }
    }
    __device__ double score(float x) const { return SIGMOID ? sigmoid64(x) : exp(static_cast<double>(x) - base) / sum; }
    __device__ double key(float x, int e) const
    {
        const double k = SCORES && bias != nullptr ? score(x) + bias[e] : x;
        return x > -INFINITY && k > -INFINITY ? k : -INFINITY;
    }
};

// Whether this lane's group (by parts) stays, by values in 64 bits.
template <int V, int P, int L, bool SIGMOID, bool SCORES>
__device__ __forceinline__ bool group_stays_exactly(const float* bias, const float* token, int E, int groups, int top_groups, int group_best, int first, float base)
{
    const int in = lane_id() % L;
    const GroupParts<L> g(E, groups, in);
    const ExactKeys<V, P, L, SIGMOID, SCORES> keys(bias, token, first, base);
    double a = -INFINITY, b = -INFINITY;
#pragma unroll 1
    for (int e = g.begin; e < g.end; ++e) {
        double s = keys.key(token[e], e);
        if (SCORES && bias == nullptr && s > -INFINITY) s = keys.score(token[e]);
        b = fmax(b, fmin(a, s));
        a = fmax(a, s);
    }
    for (int off = 1; off < g.parts; off *= 2) {
        const double a2 = __shfl_xor(a, off, kWave), b2 = __shfl_xor(b, off, kWave);
        b = fmax(fmax(b, b2), fmin(a, a2));
        a = fmax(a, a2);
    }
    if (group_best == 2 && b > -INFINITY) a += b;
    int ahead = 0;
#pragma unroll 1
    for (int i = 0; i < groups; ++i) {
        const double other = __shfl(a, (lane_id() & ~(L - 1)) + i * g.parts, kWave);
        ahead += other > a || (other == a && i < g.mine) ? 1 : 0;
    }
    return ahead < top_groups && a > -INFINITY;
}

__device__ __forceinline__ int id_of(uint32_t n) { return (1 << kIdBits) - 1 - static_cast<int>(n & ((1u << kIdBits) - 1u)); }

// Candidates, one a lane (0: none), in the order of their keys in 64 bits.
template <int V, int P, int L, bool SIGMOID, bool SCORES>
__device__ __forceinline__ uint32_t order_exactly(const float* bias, float* token, uint32_t mine, int first, float base)
{
    const int in = lane_id() % L, from = lane_id() & ~(L - 1), e = id_of(mine);
    const ExactKeys<V, P, L, SIGMOID, SCORES> keys(bias, token, first, base);
    const double exact = mine != 0u ? keys.key(token[mine != 0u ? e : 0], e) : -INFINITY;
    int ahead = 0;
#pragma unroll 4
    for (int i = 0; i < L; ++i) {
        const double other = __shfl(exact, from + i, kWave);
        const int id = __shfl(e, from + i, kWave);
        ahead += other > exact || (other == exact && id < e) ? 1 : 0;
    }
    uint32_t* order = reinterpret_cast<uint32_t*>(token);
    lds_in_order();
    order[in] = 0u;
    lds_in_order();
    if (exact > -INFINITY) order[ahead] = mine;
    lds_in_order();
    mine = order[in];
    lds_in_order();
    return mine;
}

template <int V, int P>
__device__ __forceinline__ void load_bias(const RouteCall& p, int first, float (&bias)[V])
{
    if (p.bias == nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) bias[v] = 0.0f;
    } else load_row<V, P, false>(p.bias, first, p.E, 0.0f, bias, reinterpret_cast<uintptr_t>(p.bias) % 16 == 0);
}

// `token`: room for the token's logits in LDS.  sure: whether the lane's part of the choice is the definition's.
template <int V, int P, int L, bool BF16, bool SIGMOID, bool SCORES, bool GROUPS>
__device__ __forceinline__ int choose_by_classes(const RouteCall& p, const void* row, float (&l)[V], float (&bias)[V], float* token, int first, int in, float base,
                                                 float inverse, bool& sure)
{
    auto score = [&](float v) {
        if constexpr (SIGMOID) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504f));
        else return __builtin_amdgcn_exp2f((v - base) * 1.44269504f) * inverse;
    };
    uint32_t key[V];
    sure = true;
    float apart = 0.0f;  // classes that are no further apart say nothing
    Classes c{0.0f, 0.0f};
    // A sigmoid is off by less than 2^-21 (half a unit of 2^-23 and less from the exponent and its argument, one from the sum and two from the reciprocal), a
    // softmax by less than 2^-19 of the largest score (21 sums of terms that are off by two units each), and a sum with a bias by half a last place more.
    auto classes_of_scores = [&]() {
        float f[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            f[v] = score(l[v]);
            if (SCORES && p.bias != nullptr) f[v] += bias[v];
        }
        c = classes_of<V, L>(f);
        const float error = (SIGMOID ? 0x1p-21f : 0x1p-19f * inverse) + 0x1p-23f * fmaxf(fabsf(c.most), fabsf(c.most - kClasses * __builtin_amdgcn_rcpf(c.step)));
        apart = c.step > 0.0f ? 4.0f + 2.0f * error * c.step : 2.0f * kClasses;
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = class_of(f[v], c, l[v]);
    };
    auto classes_of_logits = [&]() {
        if constexpr (BF16) {
            apart = -1.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = ordered(l[v]);
        } else {
            c = classes_of<V, L>(l);
            apart = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = class_of(l[v], c, l[v]);
        }
    };
    if constexpr (SCORES) classes_of_scores();
    else classes_of_logits();

    unsigned long long stay = ~0ull;  // lanes whose group stays, `parts` of them a group
    int parts = 1;
    const int size = p.E / p.groups, inverse_size = ((1 << 20) + size - 1) / size;  // (e * inverse_size is less than e / size + 1 / 4 in 2^20s: floors agree up to 512)
    if constexpr (GROUPS) {
        const GroupParts<L> g(p.E, p.groups, in);
        uint32_t a = 0u, b = 0u;
        uint32_t* classes = reinterpret_cast<uint32_t*>(token);
#pragma unroll
        for (int v = 0; v < V; v += 4) *reinterpret_cast<uint4*>(classes + first + place<P>(v)) = make_uint4(key[v], key[v + 1], key[v + 2], key[v + 3]);
        lds_in_order();
        auto meet = [&](int e) {
            const uint32_t k = classes[e];
            b = max(b, min(a, k));
            a = max(a, k);
        };
        const int share = size / g.parts;
        if (share * g.parts == size && share >= 16 && (share & (share - 1)) == 0) {
            // Lanes that begin a power of two apart would all be at the same banks (groups of 32, 32768 tokens: 3.9 M cycles of conflicts, now 0.3; one token 0.6 us less):
            // each begins elsewhere in its share, those of all tokens at different ones.
            const int begin = g.mine < p.groups ? g.begin : 0, turn = (in & ~3) + lane_id() / L;
#pragma unroll 4
            for (int i = 0; i < share; ++i) meet(begin + ((i + turn) & (share - 1)));
        } else {
#pragma unroll 4
            for (int e = g.begin; e < g.end; ++e) meet(e);
        }
        if (g.parts > 1) best_two<1>(a, b);
        if (g.parts > 2) best_two<2>(a, b);
        if (g.parts > 4) best_two<4>(a, b);
        if (g.parts > 8) best_two<8>(a, b);
        if (L > 16 && g.parts > 16) best_two<16>(a, b);
        const int group = g.mine;
        const uint32_t own = group < p.groups ? (p.group_best == 2 ? a + b : a) << 6 | static_cast<uint32_t>(63 - group) : 0u;
        uint32_t left = own, last = 0u, next = 0u;
        for (int j = 0; j <= p.top_groups; ++j) {
            last = next;
            next = token_max_u32<L>(left);
            if (left == next) left = 0u;
        }
        bool stays = own >= last;
        // (a class of one may be anything below; sums of one and of two classes do not compare)
        const float gap = static_cast<float>((last >> 6) - (next >> 6)), need = p.group_best == 2 ? 2.0f * apart : apart;
        bool certain = (gap > need && (last >> 6) > 1u) || (BF16 && !SCORES);
        if (p.group_best == 2 && b <= 1u && a != 0u) certain = false;
        if (!(BF16 && !SCORES) && __ballot(!certain) != 0ull) {
            share_logits<V, P, L>(l, token, first);
            stays = group_stays_exactly<V, P, L, SIGMOID, SCORES>(p.bias, token, p.E, p.groups, p.top_groups, p.group_best, first, base);
            // (Classes and what they are made from are formed again, for what is rarely needed: held meanwhile, they cost registers always.)
            load_row<V, P, BF16>(row, first, p.E, -INFINITY, l);
            if constexpr (SCORES) load_bias<V, P>(p, first, bias), classes_of_scores();
            else classes_of_logits();
        }
        stay = __ballot(stays) >> (lane_id() & ~(L - 1));
        if (SCORES && p.bias == nullptr) classes_of_logits();
        parts = g.parts;
    }
    // in place of the experts that do not stay, nothing; classes with their ids, sorted
    auto number = [&]() {
        if constexpr (GROUPS) {
#pragma unroll
            for (int v = 0; v < V; v += 4) {
                int q = (first + place<P>(v)) * inverse_size >> 20, rest = first + place<P>(v) - q * size;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (((stay >> min(q * parts, kWave - 1)) & 1ull) == 0ull) key[v + i] = 0u;
                    if (++rest == size) ++q, rest = 0;
                }
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = key[v] != 0u ? key[v] << kIdBits | static_cast<uint32_t>((1 << kIdBits) - 1 - first - place<P>(v)) : 0u;
        sort_keys<V>(key);
    };
    uint32_t mine = 0u, next = 0u;
    // the `count` largest: the largest of all heads is taken off its lane's list, of which M places are moved
    auto take = [&](auto places, int count) {
        constexpr int M = decltype(places)::value;
        for (int j = 0; j < count; ++j) {
            next = token_max_u32<L>(key[0]);
            mine = in == j ? next : mine;
            const bool taken = key[0] == next;
#pragma unroll
            for (int v = 0; v < M; ++v) key[v] = taken ? (v + 1 < V ? key[v + 1] : 0u) : key[v];
        }
    };
    const std::integral_constant<int, V> all;
    // With M places an element past the lane's first M + 1 is that one again, at once: neighbours that are equal, and not sure.  Four are enough for all but 4e-4 of tokens
    // that choose eight of 256 (7e-4 of half of eight groups), so for all but 3e-3 of wavefronts; where nothing else is unsure, nine.
    const std::integral_constant<int, (V <= 9 ? V : BF16 && !SCORES ? 9 : 4)> some;
    number();
    if (V > 9 && p.k <= 8) take(some, p.k + 1);
    else take(all, p.k + 1);
    const uint32_t right = static_cast<uint32_t>(__shfl_down(static_cast<int>(mine), 1, kWave)), after = in == p.k - 1 ? next : right;
    const float gap = static_cast<float>(mine >> kIdBits) - static_cast<float>(after >> kIdBits);
    const bool certain = in >= p.k || mine == 0u || (mine != after && ((BF16 && p.bias == nullptr) || (gap > apart && mine >> kIdBits > 1u)));
    if (!(BF16 && !SCORES) && __ballot(!certain) != 0ull) {
        // Neighbours that classes do not tell apart: the L best by class, a lane each, put in order by their keys in 64 bits.  The k best are among them if the
        // last one is clearly behind the k-th, or there are no more.
        const uint32_t behind_all = next;
        load_row<V, P, BF16>(row, first, p.E, -INFINITY, l);
        if constexpr (SCORES) load_bias<V, P>(p, first, bias);
        if (SCORES && p.bias != nullptr) classes_of_scores();
        else classes_of_logits();
        number();
        mine = 0u;
        take(all, L);
        const int from = lane_id() & ~(L - 1);
        const uint32_t kth = static_cast<uint32_t>(__shfl(static_cast<int>(mine), from + p.k - 1, kWave)) >> kIdBits;
        const uint32_t end = static_cast<uint32_t>(__shfl(static_cast<int>(mine), from + L - 1, kWave)) >> kIdBits;
        const uint32_t behind = p.k == L ? behind_all >> kIdBits : end;
        sure = behind == 0u || kth == 0u || (static_cast<float>(kth) - static_cast<float>(behind) > apart && kth > 1u);
        share_logits<V, P, L>(l, token, first);
        mine = order_exactly<V, P, L, SIGMOID, SCORES>(p.bias, token, mine, first, base);
    }
    return in < p.k && mine != 0u ? id_of(mine) : -1;
}

template <int V, int L, bool BF16, bool SIGMOID, bool SCORES, bool GROUPS>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(const RouteCall p)
{
    __shared__ double keys[V * kRouteThreads];  // of the exact choice, or a token's logits or classes
    constexpr int P = 4 * L;
    const int in = lane_id() % L, first = in * 4;
    constexpr int kTokens = kRouteThreads / L;
    const bool by_classes = !GROUPS || p.groups <= L;
    double* mine_in_lds = keys + threadIdx.x / kWave * (V * kWave);
    float* token = reinterpret_cast<float*>(mine_in_lds) + lane_id() / L * (L * V);
    const int64_t t0 = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * kTokens;
    if (t0 >= p.T) return;
    const int64_t t = t0 + threadIdx.x / L;
    const bool there = t < p.T;
    const int64_t row = min(t, p.T - 1);
    const void* at = row_at<BF16>(p.logits, row * p.E);
    float l[V], bias[V];
    load_row<V, P, BF16>(at, first, p.E, -INFINITY, l);
    if constexpr (SCORES) load_bias<V, P>(p, first, bias);
    float most = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        most = fmaxf(most, l[v]);  // (ignores a NaN)
        nan |= l[v] != l[v];
    }
    most = token_max<L>(most);
    const bool broken = (__ballot(nan) >> (lane_id() & ~(L - 1)) & ((1ull << L) - 1ull)) != 0ull || (!SIGMOID && most == INFINITY);
    const float base = most == -INFINITY ? 0.0f : most;
    const bool share = p.renormalize && p.k > 1;
    float sum = 0.0f;
    if (!SIGMOID && (SCORES || !share || p.scores != nullptr)) {
#pragma unroll
        for (int v = 0; v < V; ++v) sum += exp_below(l[v] - base);
        sum = token_sum<L>(sum);
    }
    const float inverse = 1.0f / sum;
    if (p.scores != nullptr && there) {
        float s[V];
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = SIGMOID ? sigmoid(l[v]) : (most == -INFINITY ? 0.0f : exp_below(l[v] - base) * inverse);
        store_row<V, P, false>(p.scores + row * p.E, first, p.E, s);
    }
    int chosen = -1;
    bool sure = false;
    if (by_classes) chosen = choose_by_classes<V, P, L, BF16, SIGMOID, SCORES, GROUPS>(p, at, l, bias, token, first, in, base, inverse, sure);
    if ((GROUPS || !(BF16 && !SCORES)) && __ballot(!sure) != 0ull) {
        load_row<V, P, BF16>(at, first, p.E, -INFINITY, l);
        lds_in_order();  // (the place held the tokens' logits)
#pragma unroll
        for (int v = 0; v < V; ++v) mine_in_lds[v * kWave + lane_id()] = l[v];
        chosen = choose_exactly<V, P, L, SIGMOID, SCORES, GROUPS>(p, mine_in_lds + lane_id(), first, in, base);
    }
    const bool live = chosen >= 0;
    const float mine = live ? load_logit<BF16>(at, chosen) : -INFINITY;
    float w;
    if (share) w = chosen_share<L, SIGMOID>(mine, live);
    else if (!live) w = 0.0f;
    else w = SIGMOID ? sigmoid(mine) : exp_below(mine - base) * inverse;
    if (there && in < p.k) {
        p.idx[row * p.k + in] = chosen;
        p.w[row * p.k + in] = broken ? NAN : p.scale * w;
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
    __shared__ __attribute__((aligned(16))) float changes[V * kRouteThreads];
    const int lane = lane_id(), in = lane % L;
    constexpr int kTokens = kRouteThreads / L;
    const int64_t t0 = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * kTokens;
    if (t0 >= p.T) return;
    const int64_t t = t0 + threadIdx.x / L;
    const bool there = t < p.T;
    const int64_t row = min(t, p.T - 1);
    const void* at = row_at<BF16>(p.logits, row * p.E);
    constexpr int P = 4 * L;
    const int first = in * 4;
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
        load_row<V, P, BF16>(at, first, p.E, -INFINITY, l);
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = 0.0f;
        if (p.dscores != nullptr) load_row<V, P, false>(p.dscores + row * p.dscores_stride, first, p.E, 0.0f, d);
        if constexpr (!SIGMOID) {
            most = l[0];
#pragma unroll
            for (int v = 1; v < V; ++v) most = fmaxf(most, l[v]);
            most = token_max<L>(most);
            if (most == -INFINITY) most = 0.0f;
            sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[v] = exp_below(l[v] - most);
                sum += l[v];
            }
            sum = token_sum<L>(sum);
            if (sum == 0.0f) sum = 1.0f;
            const float inverse = 1.0f / sum;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[v] *= inverse;
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
        change = p.scale * g * sigmoid_slope(mine);
    } else {
        change = p.scale * g * (expf(mine - most) / sum);
        less += token_sum<L>(change);
    }
    if (!live) change = 0.0f;
    if (all) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float slope = SIGMOID ? sigmoid_slope(l[v]) : l[v];
            out[v] = slope != 0.0f ? slope * (SIGMOID ? d[v] : d[v] - less) : 0.0f;
        }
    }
    // An expert's changes, in the order of the slots; each in its place of the row in LDS, from where the expert's lane takes it.
    float mine_all = 0.0f;
    const int id = live ? e : -1;
    for (int j = 0; j < p.k; ++j) {
        const int other = __shfl(id, (lane & ~(L - 1)) + j, kWave);
        const float c = __shfl(change, (lane & ~(L - 1)) + j, kWave);
        mine_all += other == id ? c : 0.0f;
    }
    float* token = changes + threadIdx.x / L * (L * V);
#pragma unroll
    for (int v = 0; v < V; v += 4) *reinterpret_cast<float4*>(token + first + place<P>(v)) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    lds_in_order();
    if (live) token[e] = mine_all;
    lds_in_order();
#pragma unroll
    for (int v = 0; v < V; v += 4) {
        const float4 c = *reinterpret_cast<const float4*>(token + first + place<P>(v));
        out[v] += c.x, out[v + 1] += c.y, out[v + 2] += c.z, out[v + 3] += c.w;
    }
    if (there) store_row<V, P, BF16>(static_cast<uint8_t*>(p.dlogits) + row * p.E * (BF16 ? 2 : 4), first, p.E, out);
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

// (Not a loop over the tokens: what the rare paths need would be made ready in front of it.)
static dim3 route_grid(int64_t T, int tokens)
{
    const int64_t blocks = (T + tokens - 1) / tokens, wide = blocks < (1 << 20) ? blocks : 1 << 20;
    return dim3(static_cast<unsigned>(wide), static_cast<unsigned>((blocks + wide - 1) / wide));
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
    const bool in_groups = p.groups > 1, by_scores = bias != nullptr || (in_groups && group_best == 2);
    pick_route(E, dt, score, [&](auto v, auto l, auto bf16, auto sigmoid) {
        constexpr int kTokens = kRouteThreads / decltype(l)::value;
        auto launch = [&](auto scores, auto grouped) {
            hipLaunchKernelGGL((route_kernel<decltype(v)::value, decltype(l)::value, decltype(bf16)::value, decltype(sigmoid)::value, decltype(scores)::value, decltype(grouped)::value>),
                               route_grid(T, kTokens), dim3(kRouteThreads), 0, static_cast<hipStream_t>(stream), p);
        };
        const std::true_type yes;
        const std::false_type no;
        if (by_scores) in_groups ? launch(yes, yes) : launch(yes, no);
        else in_groups ? launch(no, yes) : launch(no, no);
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
                           route_grid(T, kTokens), dim3(kRouteThreads), 0, static_cast<hipStream_t>(stream), p);
    });
    return check_launch(fn);
}
