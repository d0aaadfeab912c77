// q4_quantize, q4_dequantize: rows in groups of 32, 64 or 128 4-bit integers with a common scale and zero point.  Pure streams: a lane takes eight
// elements, 4, 8 or 16 lanes a group.
#include "q4.hpp"

namespace exf {

// Reductions over the LANES lanes of a group, in every lane: inside quads, then of a row's halves and of a row of 16 mirrored.
template <int LANES, class F>
__device__ __forceinline__ uint32_t over_group(uint32_t v, F f)
{
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true));   // quad_perm 1,0,3,2
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true));   // quad_perm 2,3,0,1
    if constexpr (LANES >= 8) v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true));   // row_half_mirror
    if constexpr (LANES >= 16) v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true));  // row_mirror
    return v;
}

// x / 15 or x / 7 in 64 bits, correctly rounded: by a reciprocal, its remainder put back (as Markstein does).
template <int BY>
__device__ __forceinline__ double divided(double x)
{
    constexpr double r = 1.0 / BY;
    const double q = x * r;
    return fma(fma(static_cast<double>(-BY), q, x), r, q);
}

// The integer nearest to x / s, halfway the even one, |x / s| < 2^20, s from 2^-90 to 2^126, `inverse` 1 / s to a unit.
//   bf16: x - h s for an h between two integers is 0 or more than a 2^-15th of x, and what is left of x put back makes h of a quotient that is h.
//   fp32: q is off by one at most where the quotient is next to the middle between two integers, and there x - q s is exact (a multiple of half the last place of s,
// below 2 s).
template <bool BF16>
__device__ __forceinline__ float nearest_quotient(float x, float s, float inverse)
{
    if constexpr (BF16) {
        const float t = x * inverse;
        return rintf(fmaf(fmaf(-t, s, x), inverse, t));
    } else {
        float q = rintf(x * inverse);
        const float rest = fmaf(-q, s, x), half = 0.5f * s;
        const bool odd = (static_cast<int>(q) & 1) != 0;
        if (rest > half || (rest == half && odd)) q += 1.0f;
        else if (rest < -half || (rest == -half && odd)) q -= 1.0f;
        return q;
    }
}

// The least value of a group and 0, the largest and 0, and whether it holds an infinity or a NaN.  By the bits: of numbers with a sign the one further from zero
// has the larger bits, and with those of a sign the largest bits as a whole number without a sign are the least value.
struct Ends {
    float lo, hi;
    bool broken;
};
typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2_t;
typedef __attribute__((__vector_size__(2 * sizeof(int16_t)))) int16_t i16x2_t;
__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b)
{
    u16x2_t p, q;
    __builtin_memcpy(&p, &a, 4), __builtin_memcpy(&q, &b, 4);
    p = __builtin_elementwise_max(p, q);
    __builtin_memcpy(&a, &p, 4);
    return a;
}
__device__ __forceinline__ uint32_t max_i16(uint32_t a, uint32_t b)
{
    i16x2_t p, q;
    __builtin_memcpy(&p, &a, 4), __builtin_memcpy(&q, &b, 4);
    p = __builtin_elementwise_max(p, q);
    __builtin_memcpy(&a, &p, 4);
    return a;
}
template <bool BF16, int LANES>
__device__ __forceinline__ Ends ends_of_group(const uint4 (&raw)[BF16 ? 1 : 2])
{
    uint32_t hi, lo;  // bits of the largest, 0 at least; of the least, below 2^31 (2^15) if there is none below 0
    if constexpr (BF16) {
        const uint4 t = raw[0];
        uint32_t h = max_i16(max_i16(max_i16(t.x, t.y), max_i16(t.z, t.w)), 0u), l = max_u16(max_u16(t.x, t.y), max_u16(t.z, t.w));
        h = max_u16(h, h >> 16), l = max_u16(l, l >> 16);
        const uint32_t both = over_group<LANES>((l << 16) | (h & 0xffffu), [](uint32_t a, uint32_t b) { return max_u16(a, b); });
        hi = both << 16, lo = both & 0xffff0000u;
    } else {
        const uint4 a = raw[0], b = raw[1];
        auto largest = [](int32_t p, int32_t q) { return max(p, q); };
        int32_t h = largest(largest(largest(a.x, a.y), largest(a.z, a.w)), largest(largest(b.x, b.y), largest(b.z, b.w)));
        uint32_t l = max(max(max(a.x, a.y), max(a.z, a.w)), max(max(b.x, b.y), max(b.z, b.w)));
        hi = over_group<LANES>(static_cast<uint32_t>(max(h, 0)), [](uint32_t p, uint32_t q) { return max(p, q); });
        lo = over_group<LANES>(l, [](uint32_t p, uint32_t q) { return max(p, q); });
    }
    Ends r;
    r.broken = hi >= 0x7f800000u || lo >= 0xff800000u;
    r.hi = __uint_as_float(hi);
    r.lo = lo >= 0x80000000u ? __uint_as_float(lo) : 0.0f;
    return r;
}

constexpr int kQ4Pieces = 4;  // of a lane on their way

// What bounds it: HBM, and the vector instructions next to it.  2^29 bf16 values in groups of 128 with zero points (1.36 GB) 241 us, 5.6 TB/s; with a piece a lane
// at a time, ties decided by the remainder, ends by floating-point comparisons and codes packed one by one 430.
template <bool BF16, int GROUP, bool ZERO, int U>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const void* __restrict__ x, int64_t pieces, uint32_t* __restrict__ q, void* __restrict__ scale,
                                                          uint8_t* __restrict__ zero)
{
    constexpr int LANES = GROUP / 8;
    // (groups are whole, and so are the lanes that hold one)
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * 256 * U + threadIdx.x; i0 < pieces; i0 += static_cast<int64_t>(gridDim.x) * 256 * U) {
        // (past the last piece the last one again, in groups of its own, and not stored)
        uint4 raw[U][BF16 ? 1 : 2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < (BF16 ? 1 : 2); ++h) raw[u][h] = load_stream16(static_cast<const uint4*>(x) + min(i0 + u * 256, pieces - 1) * (BF16 ? 1 : 2) + h);
        Ends ends[U];
        float s[U], by[U];
        bool rare = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ends[u] = ends_of_group<BF16, LANES>(raw[u]);
            const float hi = ends[u].hi, lo = ends[u].lo;
            if constexpr (ZERO) s[u] = static_cast<float>(divided<15>(static_cast<double>(hi) - static_cast<double>(lo)));
            else s[u] = static_cast<float>(divided<7>(static_cast<double>(hi > -lo ? hi : -lo)));
            if constexpr (BF16) s[u] = __uint_as_float(pack_bf16x2(s[u], s[u]) << 16);
            by[u] = s[u] == 0.0f ? 1.0f : s[u];  // (then all quotients round to 0)
            rare |= ends[u].broken || by[u] < 0x1p-90f;
        }
        const bool some_rare = __ballot(rare) != 0ull;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8], lo = ends[u].lo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (BF16) {
                    const uint32_t w = j == 0 ? raw[u][0].x : j == 1 ? raw[u][0].y : j == 2 ? raw[u][0].z : raw[u][0].w;
                    v[2 * j] = __uint_as_float(w << 16), v[2 * j + 1] = __uint_as_float(w & 0xffff0000u);
                } else {
                    const uint4 t = raw[u][j / 2];
                    v[2 * j] = __uint_as_float(j % 2 == 0 ? t.x : t.z), v[2 * j + 1] = __uint_as_float(j % 2 == 0 ? t.y : t.w);
                }
            }
            if (some_rare) {
                // an infinity or a NaN: all of the group stands for NaN; small scales: both sides of the quotient multiplied by a power of two, exactly
                const bool broken = ends[u].broken;
                const float up = broken ? 0.0f : (by[u] < 0x1p-90f ? 0x1p64f : 1.0f);
                s[u] = broken ? __uint_as_float(0x7fc00000u) : s[u];
                by[u] = broken ? 1.0f : by[u] * up;
                lo = broken ? 0.0f : lo * up;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = broken ? 0.0f : v[j] * up;
            }
            const float inverse = __builtin_amdgcn_rcpf(by[u]);
            float at = 8.0f;
            if constexpr (ZERO) at = __builtin_amdgcn_fmed3f(nearest_quotient<BF16>(-lo, by[u], inverse), 0.0f, 15.0f);
            float c[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] = __builtin_amdgcn_fmed3f(nearest_quotient<BF16>(v[j], by[u], inverse) + at, 0.0f, 15.0f);
            auto four = [](float a, float b, float c, float d) { return static_cast<uint32_t>(fmaf(fmaf(fmaf(d, 16.0f, c), 16.0f, b), 16.0f, a)); };
            const int64_t i = i0 + u * 256;
            if (i >= pieces) continue;
            __builtin_nontemporal_store(four(c[0], c[1], c[2], c[3]) | four(c[4], c[5], c[6], c[7]) << 16, q + i);
            if (threadIdx.x % LANES == 0) {
                const int64_t g = i / LANES;
                if constexpr (BF16) static_cast<bf16_t*>(scale)[g] = static_cast<bf16_t>(__float_as_uint(s[u]) >> 16);
                else static_cast<float*>(scale)[g] = s[u];
                if constexpr (ZERO) zero[g] = static_cast<uint8_t>(at);
            }
        }
    }
}

// A lane writes 16 bytes: eight elements in bf16, four in fp32 (neighbouring lanes write what lies together: with eight 170 us for 2^27 values, now 118).
template <bool BF16, int GROUP, int U>
__global__ __launch_bounds__(256) void q4_dequantize_kernel(const uint32_t* __restrict__ q, const void* __restrict__ scale, const uint8_t* __restrict__ zero,
                                                            int64_t pieces, uint4* __restrict__ out)
{
    constexpr int N = BF16 ? 8 : 4;  // elements of a piece
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * 256 * U + threadIdx.x; i0 < pieces; i0 += static_cast<int64_t>(gridDim.x) * 256 * U) {
        uint32_t code[U], s4[U], z4[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = min(i0 + u * 256, pieces - 1), g = i / (GROUP / N);
            code[u] = BF16 ? __builtin_nontemporal_load(q + i) : static_cast<uint32_t>(__builtin_nontemporal_load(reinterpret_cast<const uint16_t*>(q) + i));
            s4[u] = BF16 ? static_cast<uint32_t>(static_cast<const bf16_t*>(scale)[g]) << 16 : static_cast<const uint32_t*>(scale)[g];
            z4[u] = zero != nullptr ? zero[g] : 8u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * 256;
            if (i >= pieces) continue;
            const float s = __uint_as_float(s4[u]), at = static_cast<float>(z4[u]);
            const uint32_t even = code[u] & 0x0f0f0f0fu, odd = (code[u] >> 4) & 0x0f0f0f0fu;
            float v[N];
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                v[2 * j] = (static_cast<float>((even >> (8 * j)) & 255u) - at) * s;
                v[2 * j + 1] = (static_cast<float>((odd >> (8 * j)) & 255u) - at) * s;
            }
            if constexpr (BF16) store_stream16(out + i, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
            else store_stream16(out + i, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
        }
    }
}

static int check_q4(const char* fn, const void* x, int64_t rows, int k, int group, int dt, const uint8_t* q, const void* scale, const uint8_t* zero)
{
    if (dt != EXF_F32 && dt != EXF_BF16) return fail(EXF_ERR_BAD_DTYPE, "%s: dt = %d", fn, dt);
    if (int rc = check_q4_group(fn, k, group)) return rc;
    if (rows < 0 || rows >= (1ll << 40) / k) return fail(EXF_ERR_BAD_SHAPE, "%s: rows = %lld outside [0, 2^40 / k)", fn, static_cast<long long>(rows));
    if (rows == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, x);
    EXF_CHECK_PTR(fn, q);
    EXF_CHECK_PTR(fn, scale);
    EXF_CHECK_ALIGNED(fn, x);
    EXF_CHECK_ALIGNED(fn, q);
    EXF_CHECK_ALIGNED(fn, scale);
    if (int rc = check_q4_zero(fn, zero, dt)) return rc;
    const size_t n = static_cast<size_t>(rows) * k, el = dt == EXF_BF16 ? 2 : 4, groups = n / group;
    const struct {
        const void* at;
        size_t bytes;
    } all[] = {{x, n * el}, {q, n / 2}, {scale, groups * el}, {zero, groups}};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(all[i].at, all[i].bytes, all[j].at, all[j].bytes)) return fail(EXF_ERR_BAD_SHAPE, "%s: the arrays must not overlap", fn);
    return EXF_OK;
}

// Pieces of a lane: one where that leaves less than eight wavefronts a SIMD.  One and four, us: 2^22 fp32 values 6.5 and 8.0 (back 7.1 and 8.4), bf16 5.4 and 5.7; 2^24
// bf16 12.1 and 11.8 (13.9 and 11.3); 2^27 65 and 59 (83 and 64).
static bool few_pieces(int64_t pieces) { return pieces < 8ll * 1024 * kWave * kQ4Pieces; }
static dim3 pieces_grid(int64_t pieces, int of_a_lane)
{
    const int64_t blocks = (pieces + 256 * of_a_lane - 1) / (256 * of_a_lane);
    return dim3(static_cast<unsigned>(blocks < (1 << 22) ? blocks : 1 << 22));
}

}  // namespace exf

extern "C" int q4_quantize(const void* x, int64_t rows, int k, int group, int dt, uint8_t* q, void* scale, uint8_t* zero, void* stream)
{
    using namespace exf;
    if (int rc = check_q4("q4_quantize", x, rows, k, group, dt, q, scale, zero)) return rc;
    if (rows == 0) return EXF_OK;
    const int64_t pieces = rows * k / 8;
    pick_q4_group(group, [&](auto size) {
        auto run = [&](auto bf16, auto with_zero, auto of_a_lane) {
            constexpr int U = decltype(of_a_lane)::value;
            hipLaunchKernelGGL((q4_quantize_kernel<decltype(bf16)::value, decltype(size)::value, decltype(with_zero)::value, U>), pieces_grid(pieces, U), dim3(256), 0,
                               static_cast<hipStream_t>(stream), x, pieces, reinterpret_cast<uint32_t*>(q), scale, zero);
        };
        auto with = [&](auto bf16, auto with_zero) {
            if (few_pieces(pieces)) run(bf16, with_zero, std::integral_constant<int, 1>());
            else run(bf16, with_zero, std::integral_constant<int, kQ4Pieces>());
        };
        const std::true_type yes;
        const std::false_type no;
        if (dt == EXF_BF16) zero != nullptr ? with(yes, yes) : with(yes, no);
        else zero != nullptr ? with(no, yes) : with(no, no);
    });
    return check_launch("q4_quantize");
}

extern "C" int q4_dequantize(const uint8_t* q, const void* scale, const uint8_t* zero, int64_t rows, int k, int group, int dt, void* out, void* stream)
{
    using namespace exf;
    if (int rc = check_q4("q4_dequantize", out, rows, k, group, dt, q, scale, zero)) return rc;
    if (rows == 0) return EXF_OK;
    const int64_t pieces = rows * k / (dt == EXF_BF16 ? 8 : 4);
    pick_q4_group(group, [&](auto size) {
        auto run = [&](auto bf16, auto of_a_lane) {
            constexpr int U = decltype(of_a_lane)::value;
            hipLaunchKernelGGL((q4_dequantize_kernel<decltype(bf16)::value, decltype(size)::value, U>), pieces_grid(pieces, U), dim3(256), 0,
                               static_cast<hipStream_t>(stream), reinterpret_cast<const uint32_t*>(q), scale, zero, pieces, static_cast<uint4*>(out));
        };
        auto with = [&](auto bf16) {
            if (few_pieces(pieces)) run(bf16, std::integral_constant<int, 1>());
            else run(bf16, std::integral_constant<int, kQ4Pieces>());
        };
        if (dt == EXF_BF16) with(std::true_type());
        else with(std::false_type());
    });
    return check_launch("q4_dequantize");
}
