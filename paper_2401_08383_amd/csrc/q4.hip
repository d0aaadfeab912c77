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

// The integer nearest to x / s, halfway the even one, |x / s| < 2^20, s > 2^-126.  q is off by one at most where the quotient is next to the middle
// between two integers, and there x - q s is exact (a multiple of half the last place of s, below 2 s).
__device__ __forceinline__ float nearest_quotient(float x, float s, float inverse)
{
    float q = rintf(x * inverse);
    const float rest = fmaf(-q, s, x), half = 0.5f * s;
    const bool odd = (static_cast<int>(q) & 1) != 0;
    if (rest > half || (rest == half && odd)) q += 1.0f;
    else if (rest < -half || (rest == -half && odd)) q -= 1.0f;
    return q;
}

template <bool BF16, int GROUP, bool ZERO>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const void* __restrict__ x, int64_t pieces, uint32_t* __restrict__ q, void* __restrict__ scale,
                                                          uint8_t* __restrict__ zero)
{
    constexpr int LANES = GROUP / 8;
    const int64_t step = static_cast<int64_t>(gridDim.x) * 256;
    // (groups are whole, and so are the lanes that hold one)
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += step) {
        uint32_t bits[8];
        load_bits8<BF16>(static_cast<const uint8_t*>(x) + i * (BF16 ? 16 : 32), bits);
        float lo = 0.0f, hi = 0.0f;
        uint32_t largest = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo = fminf(lo, __uint_as_float(bits[j]));
            hi = fmaxf(hi, __uint_as_float(bits[j]));
            largest = max(largest, bits[j] & 0x7fffffffu);
        }
        largest = over_group<LANES>(largest, [](uint32_t a, uint32_t b) { return max(a, b); });
        float s;
        if constexpr (ZERO) {
            lo = __uint_as_float(over_group<LANES>(__float_as_uint(lo), [](uint32_t a, uint32_t b) { return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b))); }));
            hi = __uint_as_float(over_group<LANES>(__float_as_uint(hi), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
            s = static_cast<float>((static_cast<double>(hi) - static_cast<double>(lo)) / 15.0);
        } else {
            s = static_cast<float>(static_cast<double>(__uint_as_float(largest)) / 7.0);
        }
        if constexpr (BF16) s = bf16_to_f32(f32_to_bf16(s));
        const bool broken = largest >= 0x7f800000u;  // an infinity or a NaN: all of the group stands for NaN
        const bool none = broken || s == 0.0f;
        // small scales: both sides of the quotient multiplied by a power of two, exactly
        const float up = s < 0x1p-90f ? 0x1p64f : 1.0f, by = none ? 1.0f : s * up, inverse = 1.0f / by;
        const float at = ZERO ? (none ? 0.0f : fminf(nearest_quotient(-lo * up, by, inverse), 15.0f)) : 8.0f;
        uint32_t code = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float c = none ? at : fminf(fmaxf(nearest_quotient(__uint_as_float(bits[j]) * up, by, inverse) + at, 0.0f), 15.0f);
            code |= static_cast<uint32_t>(c) << (4 * j);
        }
        q[i] = code;
        if (threadIdx.x % LANES == 0) {
            const int64_t g = i / LANES;
            if (broken) s = __uint_as_float(0x7fc00000u);
            if constexpr (BF16) static_cast<bf16_t*>(scale)[g] = f32_to_bf16(s);
            else static_cast<float*>(scale)[g] = s;
            if constexpr (ZERO) zero[g] = static_cast<uint8_t>(at);
        }
    }
}

template <bool BF16, int GROUP>
__global__ __launch_bounds__(256) void q4_dequantize_kernel(const uint32_t* __restrict__ q, const void* __restrict__ scale, const uint8_t* __restrict__ zero,
                                                            int64_t pieces, uint4* __restrict__ out)
{
    const int64_t step = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += step) {
        const int64_t g = i / (GROUP / 8);
        const float s = BF16 ? bf16_to_f32(static_cast<const bf16_t*>(scale)[g]) : static_cast<const float*>(scale)[g];
        const float at = zero != nullptr ? static_cast<float>(zero[g]) : 8.0f;
        const uint32_t code = q[i];
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (static_cast<float>((code >> (4 * j)) & 15u) - at) * s;
        if constexpr (BF16) {
            store_stream16(out + i, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
        } else {
            store_stream16(out + 2 * i, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
            store_stream16(out + 2 * i + 1, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
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
    if (zero != nullptr) EXF_CHECK_ALIGNED(fn, zero);
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

static unsigned pieces_grid(int64_t pieces)
{
    const int64_t blocks = (pieces + 255) / 256;
    return static_cast<unsigned>(blocks < 4 * kStreamWorkgroups ? blocks : 4 * kStreamWorkgroups);
}

}  // namespace exf

extern "C" int q4_quantize(const void* x, int64_t rows, int k, int group, int dt, uint8_t* q, void* scale, uint8_t* zero, void* stream)
{
    using namespace exf;
    if (int rc = check_q4("q4_quantize", x, rows, k, group, dt, q, scale, zero)) return rc;
    if (rows == 0) return EXF_OK;
    const int64_t pieces = rows * k / 8;
    pick_q4_group(group, [&](auto size) {
        auto run = [&](auto bf16, auto with_zero) {
            hipLaunchKernelGGL((q4_quantize_kernel<decltype(bf16)::value, decltype(size)::value, decltype(with_zero)::value>), dim3(pieces_grid(pieces)), dim3(256), 0,
                               static_cast<hipStream_t>(stream), x, pieces, reinterpret_cast<uint32_t*>(q), scale, zero);
        };
        const std::true_type yes;
        const std::false_type no;
        if (dt == EXF_BF16) zero != nullptr ? run(yes, yes) : run(yes, no);
        else zero != nullptr ? run(no, yes) : run(no, no);
    });
    return check_launch("q4_quantize");
}

extern "C" int q4_dequantize(const uint8_t* q, const void* scale, const uint8_t* zero, int64_t rows, int k, int group, int dt, void* out, void* stream)
{
    using namespace exf;
    if (int rc = check_q4("q4_dequantize", out, rows, k, group, dt, q, scale, zero)) return rc;
    if (rows == 0) return EXF_OK;
    const int64_t pieces = rows * k / 8;
    pick_q4_group(group, [&](auto size) {
        auto run = [&](auto bf16) {
            hipLaunchKernelGGL((q4_dequantize_kernel<decltype(bf16)::value, decltype(size)::value>), dim3(pieces_grid(pieces)), dim3(256), 0,
                               static_cast<hipStream_t>(stream), reinterpret_cast<const uint32_t*>(q), scale, zero, pieces, static_cast<uint4*>(out));
        };
        if (dt == EXF_BF16) run(std::true_type());
        else run(std::false_type());
    });
    return check_launch("q4_dequantize");
}
