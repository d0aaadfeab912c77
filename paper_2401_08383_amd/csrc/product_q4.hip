// moe_grouped_product_q4: rows in bf16 or fp32 times weights in 4-bit integers with group scales.
//
// A wavefront computes 16 rows x 16 columns; the wavefronts of a workgroup share the reduction, 128 elements at a time, and join their sums through
// LDS in a fixed order.  A lane holds 32 consecutive codes of its column, 16 bytes; four lanes (quads of the matrix instruction) the 128.
//   bf16: a code becomes the number 16 + code, exactly, by putting its bits into the mantissa of 16; the matrix cores sum x (16 + code) and x over a
// group, and scale * (sum x (16 + code) - (16 + zero) sum x) joins the column's sum.
//   fp32: code - zero, exactly; the scale multiplies a group's sum.
// Groups of less than 128 elements: the codes are turned among the four quads first, so that a matrix instruction sees 32 consecutive elements.
#include "q4.hpp"

namespace exf {

constexpr int kQ4Waves = 4, kQ4Step = 128;

__device__ __forceinline__ void turn_quads(uint32_t (&r)[4])
{
    const auto a = __builtin_amdgcn_permlane32_swap(r[0], r[2], false, false), b = __builtin_amdgcn_permlane32_swap(r[1], r[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    r[0] = c[0], r[1] = c[1], r[2] = d[0], r[3] = d[1];
}

__device__ __forceinline__ bf16x8_t as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const u32x4_v v = {a, b, c, d};
    bf16x8_t r;
    __builtin_memcpy(&r, &v, sizeof(r));
    return r;
}
// Eight codes as bf16 numbers 16 + code, in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ bf16x8_t codes_bf16(uint32_t q)
{
    constexpr uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
    return as_bf16x8(((q << 3) & mask) | sixteen, ((q >> 1) & mask) | sixteen, ((q >> 5) & mask) | sixteen, ((q >> 9) & mask) | sixteen);
}
// Eight bf16 numbers in that order.
__device__ __forceinline__ bf16x8_t in_code_order(uint4 x)
{
    auto low = [](uint32_t a, uint32_t b) { return (a & 0xffffu) | (b << 16); };
    auto high = [](uint32_t a, uint32_t b) { return (a >> 16) | (b & 0xffff0000u); };
    return as_bf16x8(low(x.x, x.z), high(x.x, x.z), low(x.y, x.w), high(x.y, x.w));
}

template <bool BF16, int GROUP>
__global__ __launch_bounds__(kQ4Waves* kWave) void q4_product_kernel(const Q4Product p, int col_tiles)
{
    __shared__ f32x4_t part[kQ4Waves][kWave];
    constexpr int kGroups = kQ4Step / GROUP;     // of a step
    constexpr bool TURN = GROUP < kQ4Step;
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + 15) / 16, upto = wave_inclusive_scan(tiles);
    const int lane = lane_id(), in16 = lane & 15, quad = lane >> 4, wave = threadIdx.x / kWave;
    for (int64_t tile = blockIdx.x;; tile += gridDim.x) {
    const int row_tile = static_cast<int>(tile / col_tiles), col0 = static_cast<int>(tile % col_tiles) * 16;
    const unsigned long long owner = __ballot(row_tile < upto);
    if (owner == 0ull) return;  // (the same for all wavefronts)
    const int e = __builtin_ctzll(owner), lo = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * 16;
    const int rows = min(16, wave_read_lane(range.hi, e) - lo);
    const int64_t N = p.N, col = e * N + min(col0 + in16, p.N - 1), row = lo + min(in16, rows - 1), groups = p.K / GROUP;
    f32x4_t total = {0.f, 0.f, 0.f, 0.f};
    for (int step = wave; step * kQ4Step < p.K; step += kQ4Waves) {
        const int k0 = step * kQ4Step, codes_at = min(k0 + quad * 32, p.K - 32);
        const uint4 w4 = *reinterpret_cast<const uint4*>(p.weight + col * (p.K / 2) + codes_at / 2);
        uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        if constexpr (TURN) turn_quads(w);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int64_t i = col * groups + min(k0 / GROUP + g, static_cast<int>(groups) - 1);
            const float s = BF16 ? bf16_to_f32(static_cast<const bf16_t*>(p.scale)[i]) : static_cast<const float*>(p.scale)[i];
            const float zero = p.zero != nullptr ? static_cast<float>(p.zero[i]) : 8.0f;
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f}, sum_x = {0.f, 0.f, 0.f, 0.f};
            if (k0 + g * GROUP >= p.K) continue;  // (the last step of a row of less)
#pragma unroll
            for (int m = 0; m < GROUP / 32; ++m) {
                const int s4 = g * (GROUP / 32) + m, at = TURN ? k0 + s4 * 32 + quad * 8 : k0 + quad * 32 + s4 * 8;
                if constexpr (BF16) {
                    const bf16x8_t x = in_code_order(*reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(p.rows) + row * p.K + at));
                    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, codes_bf16(w[s4]), sum, 0, 0, 0);
                    sum_x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, as_bf16x8(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), sum_x, 0, 0, 0);
                } else {
                    const float* x = static_cast<const float*>(p.rows) + row * p.K + at;
#pragma unroll
                    for (int i8 = 0; i8 < 8; ++i8)
                        sum = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i8], static_cast<float>((w[s4] >> (4 * i8)) & 15u) - zero, sum, 0, 0, 0);
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) total[q] = fmaf(s, BF16 ? fmaf(-(16.0f + zero), sum_x[q], sum[q]) : sum[q], total[q]);
        }
    }
    part[wave][lane] = total;
    __syncthreads();
    const int c = col0 + in16;
    if (wave == 0 && c < p.N) {
    total = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    float b = 0.0f;
    if (p.bias != nullptr) b = BF16 ? bf16_to_f32(static_cast<const bf16_t*>(p.bias)[e * N + c]) : static_cast<const float*>(p.bias)[e * N + c];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int r = quad * 4 + q;
        if (r >= rows) continue;
        if constexpr (BF16) static_cast<bf16_t*>(p.out)[(lo + r) * N + c] = f32_to_bf16(total[q] + b);
        else static_cast<float*>(p.out)[(lo + r) * N + c] = total[q] + b;
    }
    }
    __syncthreads();
    }
}

}  // namespace exf

extern "C" int moe_grouped_product_q4(const void* x_sorted, const int32_t* expert_offsets, const uint8_t* w, const void* w_scale, const uint8_t* w_zero,
                                      const void* bias, int64_t A, int n, int k, int group, int E_local, int dt, void* y_sorted, void* stream)
{
    using namespace exf;
    const char* fn = "moe_grouped_product_q4";
    if (int rc = check_product_sizes(fn, A, n, k, E_local, dt)) return rc;
    if (int rc = check_q4_group(fn, k, group)) return rc;
    if (A == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, x_sorted);
    EXF_CHECK_PTR(fn, expert_offsets);
    EXF_CHECK_PTR(fn, w);
    EXF_CHECK_PTR(fn, w_scale);
    EXF_CHECK_PTR(fn, y_sorted);
    EXF_CHECK_ALIGNED(fn, x_sorted);
    EXF_CHECK_ALIGNED(fn, w);
    EXF_CHECK_ALIGNED(fn, w_scale);
    EXF_CHECK_ALIGNED(fn, y_sorted);
    if (w_zero != nullptr) EXF_CHECK_ALIGNED(fn, w_zero);
    if (bias != nullptr) EXF_CHECK_ALIGNED(fn, bias);
    const size_t el = dt == EXF_BF16 ? 2 : 4, weights = static_cast<size_t>(E_local) * n, rows = A, out_bytes = rows * n * el;
    const struct {
        const void* at;
        size_t bytes;
    } in[] = {{x_sorted, rows * k * el}, {expert_offsets, static_cast<size_t>(E_local + 1) * 4}, {w, weights * k / 2}, {w_scale, weights * (k / group) * el},
              {w_zero, weights * (k / group)}, {bias, weights * el}};
    for (const auto& i : in)
        if (overlap(y_sorted, out_bytes, i.at, i.bytes)) return fail(EXF_ERR_BAD_SHAPE, "%s: the result must not overlap an input", fn);
    const Q4Product p{x_sorted, expert_offsets, w, w_scale, w_zero, bias, y_sorted, static_cast<int>(A), k, n, E_local};
    const int64_t cols = (n + 15) / 16, grid = (A / 16 + (A < E_local ? A : E_local)) * cols;
    pick_q4_group(group, [&](auto size) {
        auto run = [&](auto bf16) {
            hipLaunchKernelGGL((q4_product_kernel<decltype(bf16)::value, decltype(size)::value>), dim3(static_cast<unsigned>(grid < (1 << 22) ? grid : 1 << 22)), dim3(kQ4Waves * kWave), 0,
                               static_cast<hipStream_t>(stream), p, static_cast<int>(cols));
        };
        if (dt == EXF_BF16) run(std::true_type());
        else run(std::false_type());
    });
    return check_launch(fn);
}
