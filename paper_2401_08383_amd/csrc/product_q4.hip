// moe_grouped_product_q4: rows in bf16 or fp32 times weights in 4-bit integers with group scales.  The mathematics, and the kernel of small products and of fp32;
// bf16 weights that fill the chip go through LDS (product_q4_stream.hip).
//
// A matrix instruction computes 16 rows x 16 columns of 32 elements of the reduction.  A lane holds 32 consecutive codes of its column, 16 bytes; the four lanes
// of a column (the quads of the instruction) 128, a step.
//   bf16: a code becomes the number 16 + code, exactly, by putting its bits into the mantissa of 16; the matrix cores sum x (16 + code) and x over a
// group, and scale * (sum x (16 + code) - (16 + zero) sum x) joins the column's sum: two fp32 roundings a group, and the sixteen costs less than three of the 24
// bits.  (128 + code takes one shift of eight codes less and six bits.)
//   fp32: code - zero, exactly; the scale multiplies a group's sum.
// The codes are turned among the quads first, so that an instruction sees 32 consecutive elements: of one group, and of rows in lines of 64 bytes.
//   Four wavefronts share the reduction of 16 rows x 16 columns, two steps each at a time (128 bytes of a column), and join their sums through LDS in a fixed
// order.  One token, 4096 x 1024: 3.9 us; one wavefront for all of the reduction 5.8, 32 columns 4.3, 64 5.4.
#include "q4.hpp"

namespace exf {

constexpr int kQ4Waves = 4, kQ4Step = 128;

template <bool BF16, int GROUP>
__global__ __launch_bounds__(kQ4Waves* kWave) void q4_product_kernel(const Q4Product p, int col_tiles)
{
    __shared__ f32x4_t part[kQ4Waves][kWave];
    constexpr int kGroups = kQ4Step / GROUP, kTurn = 4 / kGroups;  // groups of a step, steps whose groups are four
    constexpr int kPieces = BF16 ? 4 : 8;                          // 16 bytes of a row that a lane has of a step
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + 15) / 16, upto = wave_inclusive_scan(tiles);
    const int lane = lane_id(), in16 = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t N = p.N, groups = p.K / GROUP;
    const int steps = (p.K + kQ4Step - 1) / kQ4Step;
    const CodeBits bits = code_bits();
    // the wavefront's step number j, at or past `steps` where there is none
    auto step_of = [&](int j) { return (j / 2 * kQ4Waves + wave) * 2 + j % 2; };
    for (int64_t tile = blockIdx.x;; tile += gridDim.x) {
        const int row_tile = static_cast<int>(tile / col_tiles), col0 = static_cast<int>(tile % col_tiles) * 16;
        const unsigned long long owner = __ballot(row_tile < upto);
        if (owner == 0ull) return;  // (the same for all wavefronts)
        const int e = __builtin_ctzll(owner), lo = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * 16;
        const int rows = min(16, wave_read_lane(range.hi, e) - lo);
        // places that the workgroup shares, and 32-bit distances of a lane from them
        const int64_t first_col = e * N + col0;
        const global_bytes codes = shared_place(p.weight + first_col * (p.K / 2));
        const global_bytes scales = shared_place(static_cast<const uint8_t*>(p.scale) + first_col * groups * (BF16 ? 2 : 4));
        const bool has_zero = p.zero != nullptr;
        const global_bytes zeros = shared_place(has_zero ? p.zero + first_col * groups : nullptr);
        const global_bytes x = shared_place(static_cast<const uint8_t*>(p.rows) + static_cast<int64_t>(lo) * p.K * (BF16 ? 2 : 4));
        const uint32_t col = min(in16, p.N - 1 - col0), code_at = col * static_cast<uint32_t>(p.K / 2), group_at = col * static_cast<uint32_t>(groups);
        const uint32_t row_at = static_cast<uint32_t>(min(in16, rows - 1)) * p.K * (BF16 ? 2 : 4) + quad * (BF16 ? 16 : 32);
        auto load_codes = [&](int step, uint4& w) {
            if (step < steps) w = load_vector(codes + (code_at + static_cast<uint32_t>(min(step * kQ4Step + quad * 32, p.K - 32) / 2)));
        };
        auto load_rows = [&](int step, uint4 (&v)[kPieces]) {
            if (step >= steps) return;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const global_bytes at = x + min(step * kQ4Step + m * 32, p.K - 32) * (BF16 ? 2 : 4) + row_at;
                if constexpr (BF16) v[m] = load_vector(at);
                else v[2 * m] = load_vector(at), v[2 * m + 1] = load_vector(at + 16);
            }
        };
        // scales and zero points of kTurn steps of the wavefront at once, a group a quad
        auto load_scales = [&](int j, uint32_t& scale, uint32_t& zero) {
            if (step_of(j) >= steps) return;
            const uint32_t i = group_at + min(step_of(j + quad / kGroups) * kGroups + quad % kGroups, static_cast<int>(groups) - 1);
            if constexpr (BF16) scale = *reinterpret_cast<const __attribute__((address_space(1))) bf16_t*>(scales + i * 2u);
            else scale = *reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(scales + i * 4u);
            zero = has_zero ? zeros[i] : 8u;
        };
        f32x4_t total = {0.f, 0.f, 0.f, 0.f};
        auto multiply = [&](int step, const uint4& w4, const uint4 (&v)[kPieces], const float (&scale)[4], const float (&zero)[4], int first) {
            if (step >= steps) return;
            uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
            turn_quads(w);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                if (step * kQ4Step + g * GROUP >= p.K) break;  // (the last step of a row of less)
                f32x4_t sum = {0.f, 0.f, 0.f, 0.f}, sum_x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int m = g * (GROUP / 32); m < (g + 1) * (GROUP / 32); ++m) {
                    if constexpr (BF16) {
                        const bf16x8_t a = in_code_order(v[m]);
                        sum_x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, ones_bf16(), sum_x, 0, 0, 0);
                        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, codes_bf16(w[m], bits), sum, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint4 t = v[2 * m + i / 4];
                            const uint32_t element = i % 4 == 0 ? t.x : i % 4 == 1 ? t.y : i % 4 == 2 ? t.z : t.w;
                            sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(element), static_cast<float>((w[m] >> (4 * i)) & 15u) - zero[first + g], sum, 0, 0, 0);
                        }
                    }
                }
                const float less = -(16.0f + zero[first + g]);
#pragma unroll
                for (int q = 0; q < 4; ++q) total[q] = fmaf(scale[first + g], BF16 ? fmaf(less, sum_x[q], sum[q]) : sum[q], total[q]);
            }
        };
        uint4 w[4], v[2][kPieces];
        uint32_t scale_next[kGroups], zero_next[kGroups];
        load_codes(step_of(0), w[0]);
        load_codes(step_of(1), w[1]);
#pragma unroll
        for (int i = 0; i < kGroups; ++i) load_scales(i * kTurn, scale_next[i], zero_next[i]);
        load_rows(step_of(0), v[0]);
        load_rows(step_of(1), v[1]);
        for (int j0 = 0; step_of(j0) < steps; j0 += 4) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                float scale[4], zero[4];
                uint32_t s[4], z[4];
                if constexpr (BF16) {
                    spread_quads(scale_next[i] | zero_next[i] << 16, s);
#pragma unroll
                    for (int q = 0; q < 4; ++q) z[q] = s[q] >> 16, s[q] <<= 16;
                } else {
                    spread_quads(scale_next[i], s);
                    spread_quads(zero_next[i], z);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) scale[q] = __uint_as_float(s[q]), zero[q] = static_cast<float>(z[q]);
                load_scales(j0 + 4 + i * kTurn, scale_next[i], zero_next[i]);
#pragma unroll
                for (int j = 0; j < kTurn; ++j) {
                    const int u = i * kTurn + j;
                    if (u % 2 == 0) load_codes(step_of(j0 + u + 2), w[(u + 2) % 4]), load_codes(step_of(j0 + u + 3), w[(u + 3) % 4]);
                    multiply(step_of(j0 + u), w[u], v[u % 2], scale, zero, j * kGroups);
                    load_rows(step_of(j0 + u + 2), v[u % 2]);
                }
            }
        }
        part[wave][lane] = total;
        __syncthreads();
        const int c = col0 + in16;
        if (wave == 0 && c < p.N) {
            const f32x4_t sum = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
            float b = 0.0f;
            if (p.bias != nullptr) b = BF16 ? bf16_to_f32(static_cast<const bf16_t*>(p.bias)[e * N + c]) : static_cast<const float*>(p.bias)[e * N + c];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = quad * 4 + q;
                if (r >= rows) continue;
                if constexpr (BF16) static_cast<bf16_t*>(p.out)[(lo + r) * N + c] = f32_to_bf16(sum[q] + b);
                else static_cast<float*>(p.out)[(lo + r) * N + c] = sum[q] + b;
            }
        }
        __syncthreads();
    }
}

static int launch_q4_product(const Q4Product& p, int group, int dt, hipStream_t stream)
{
    const int64_t cols = (p.N + 15) / 16, grid = (p.max_rows / 16 + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
    pick_q4_group(group, [&](auto size) {
        auto run = [&](auto bf16) {
            hipLaunchKernelGGL((q4_product_kernel<decltype(bf16)::value, decltype(size)::value>), dim3(static_cast<unsigned>(grid < (1 << 22) ? grid : 1 << 22)),
                               dim3(kQ4Waves * kWave), 0, stream, p, static_cast<int>(cols));
        };
        if (dt == EXF_BF16) run(std::true_type());
        else run(std::false_type());
    });
    return EXF_OK;
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
    if (int rc = check_q4_zero(fn, w_zero, dt)) return rc;
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
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc = dt == EXF_BF16 && q4_streams(A, n, E_local) ? launch_q4_stream(p, group, s) : launch_q4_product(p, group, dt, s);
    return rc == EXF_OK ? check_launch(fn) : rc;
}
