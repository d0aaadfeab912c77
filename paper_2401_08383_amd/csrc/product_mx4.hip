// Grouped product of rows held in microscaled 4-bit floating point, on the block-scaled matrix instruction
// (v_mfma_scale_f32_16x16x128_f8f6f4): 16 x 16 outputs and 128 reduction elements at once, a lane with one block of 32 of a row, 16
// bytes, and that block's scale byte.
//
// A wavefront computes 64 x 64 outputs; operands come straight from memory.
#include <type_traits>

#include "product.hpp"

namespace exf {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4_t;
typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8_t;

constexpr int kMxTile = 64;

__device__ __forceinline__ f32x4_t mfma_mx4_direct(i32x4_t a, i32x4_t b, f32x4_t c, int scale_a, int scale_b)
{
    const i32x8_t wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};  // (4-bit operands: the lower half)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, 0, scale_a, 0, scale_b);
}

__global__ __launch_bounds__(64) void mx4_rows_kernel(const Mx4Product p, int col_tiles)
{
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + kMxTile - 1) / kMxTile;
    const int upto = wave_inclusive_scan(tiles);
    const int row_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(col_tiles)), col_tile = static_cast<int>(blockIdx.x % static_cast<unsigned>(col_tiles));
    const unsigned long long owner = __ballot(row_tile < upto);
    if (owner == 0ull) return;
    const int e = __builtin_ctzll(owner);
    const int hi = wave_read_lane(range.hi, e);
    const int row0 = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * kMxTile, col0 = col_tile * kMxTile;
    const int lane = lane_id(), in16 = lane & 15, quad = lane >> 4;
    const int64_t row_bytes = p.K / 2, N = p.N, weight_rows = static_cast<int64_t>(p.E_local) * N;
    f32x4_t acc[4][4];
    int64_t row[4], col[4];  // (rows of both arrays)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        row[i] = min(row0 + i * 16 + in16, hi - 1);
        col[i] = e * N + min(col0 + i * 16 + in16, p.N - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int blocks = p.K / 32;
    for (int b0 = 0; b0 < blocks; b0 += 4) {
        const int b = b0 + quad;
        i32x4_t fa[4], fw[4];
        int sa[4], sw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = fw[i] = i32x4_t{0, 0, 0, 0};
            sa[i] = sw[i] = 0;
            if (b < blocks) {
                fa[i] = *reinterpret_cast<const i32x4_t*>(p.rows + row[i] * row_bytes + b * 16);
                fw[i] = *reinterpret_cast<const i32x4_t*>(p.weight + col[i] * row_bytes + b * 16);
                sa[i] = p.row_scale[(static_cast<int64_t>(b / 8) * p.max_rows + row[i]) * 8 + b % 8];
                sw[i] = p.weight_scale[(b / 8 * weight_rows + col[i]) * 8 + b % 8];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma_mx4_direct(fw[j], fa[i], acc[i][j], sw[j], sa[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = row0 + i * 16 + in16, c = col0 + j * 16 + quad * 4;
            if (r >= hi || c >= p.N) continue;
            f32x4_t v = acc[i][j];
            if (p.bias != nullptr) v += *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p.bias) + e * N + c);
            *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + r * N + c) = v;
        }
}

// ---------------------------------------------------------------------------- small products
// A workgroup has 16 rows and 16 columns of one expert, its four wavefronts share the reduction and join their sums through LDS.  A lane's operand is
// one block of one row, so rows that are not held in 4 bits are quantised where they are needed, by the lane that needs them, without a
// word to any other lane: one launch instead of two, and no workspace.
//   Every 16 columns quantise the rows again, so the products are small ones, of at most kSmallTurns rows times reduction times column tiles.  One call as
// this and as two launches with a workspace, us: 490 rows over 2 of 128 x 288 8.5 and 13.0, 256 over 8 of 1024 x 1024 11.3 and 13.3, 64 over 8 of
// 1024 x 4096 (2^24) 11.1 and 14.0, of 4096 x 1024 (2^24) 14 and 14, 128 of these (2^25) 20.6 and 13.0.
constexpr int64_t kSmallTurns = 1ll << 24;
bool mx4_product_is_small(int64_t A, int n, int k) { return A <= EXF_MX4_INLINE_ROWS || (n + 15ll) / 16 <= kSmallTurns / (A * k); }

constexpr int kFewWaves = 4, kFewAhead = 2;
template <bool BF16, bool HELD>
__global__ __launch_bounds__(kFewWaves* kWave) void mx4_small_kernel(const Mx4Product p, int col_tiles)
{
    __shared__ f32x4_t part[kFewWaves][kWave];
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + 15) / 16, upto = wave_inclusive_scan(tiles);
    const int row_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(col_tiles)), col0 = static_cast<int>(blockIdx.x % static_cast<unsigned>(col_tiles)) * 16;
    const unsigned long long owner = __ballot(row_tile < upto);
    if (owner == 0ull) return;
    const int e = __builtin_ctzll(owner), lo = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * 16;
    const int rows = min(16, wave_read_lane(range.hi, e) - lo);
    const int lane = lane_id(), in16 = lane & 15, quad = lane >> 4, wave = threadIdx.x / kWave;
    const int64_t N = p.N, weight_rows = p.E_local * N, half = p.K / 2;
    const int64_t col = e * N + min(col0 + in16, p.N - 1), row = lo + min(in16, rows - 1);
    const int blocks = p.K / 32, steps = (blocks + 3) / 4;
    struct Operands {
        i32x4_t w, x;
        int sw, sx;
        uint32_t v[HELD ? 1 : 4][8];
    };
    auto load = [&](int step, Operands& o) {
        const int b = min(step * 4 + quad, blocks - 1);
        o.w = *reinterpret_cast<const i32x4_t*>(p.weight + col * half + b * 16);
        o.sw = p.weight_scale[(b / 8 * weight_rows + col) * 8 + b % 8];
        if constexpr (HELD) {
            o.x = *reinterpret_cast<const i32x4_t*>(p.rows + row * half + b * 16);
            o.sx = p.row_scale[(static_cast<int64_t>(b / 8) * p.max_rows + row) * 8 + b % 8];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) load_bits8<BF16>(p.rows + ((row * p.K + b * 32 + i * 8) * (BF16 ? 2 : 4)), o.v[i]);
        }
    };
    auto multiply = [&](int step, Operands& o, f32x4_t acc) {
        if constexpr (!HELD) {
            uint32_t largest = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) largest = max(largest, o.v[i][j] & 0x7fffffffu);
            const uint32_t byte = scale_byte(largest);
#pragma unroll
            for (int i = 0; i < 4; ++i) o.x[i] = static_cast<int>(to_codes(o.v[i], byte));
            o.sx = static_cast<int>(byte);
        }
        if (step * 4 + quad >= blocks) {  // past the end: the last block again, without a value
            o.w = o.x = i32x4_t{0, 0, 0, 0};
            o.sw = o.sx = 0;
        }
        return mfma_mx4_direct(o.w, o.x, acc, o.sw, o.sx);
    };
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    Operands o[kFewAhead];
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i) load(wave + i * kFewWaves, o[i]);
    for (int step = wave; step < steps; step += kFewAhead * kFewWaves) {
#pragma unroll
        for (int i = 0; i < kFewAhead; ++i) {
            acc = multiply(step + i * kFewWaves, o[i], acc);
            load(step + (i + kFewAhead) * kFewWaves, o[i]);
        }
    }
    part[wave][lane] = acc;
    __syncthreads();
    const int c = col0 + quad * 4;
    if (wave != 0 || in16 >= rows || c >= p.N) return;
    acc = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    if constexpr (BF16) {
        if (p.bias != nullptr)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[q] += bf16_to_f32(static_cast<const bf16_t*>(p.bias)[e * N + c + q]);
        *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + row * N + c) = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
    } else {
        if (p.bias != nullptr) acc += *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p.bias) + e * N + c);
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + row * N + c) = acc;
    }
}

int launch_mx4_small(const Mx4Product& p, int dt, hipStream_t stream)
{
    const int64_t cols = (p.N + 15) / 16, grid = (p.max_rows / 16 + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_mx4: too many tiles");
    auto run = [&](auto bf16, auto held) {
        hipLaunchKernelGGL((mx4_small_kernel<decltype(bf16)::value, decltype(held)::value>), dim3(static_cast<unsigned>(grid)), dim3(kFewWaves * kWave), 0, stream, p,
                           static_cast<int>(cols));
    };
    const std::true_type yes;
    const std::false_type no;
    if (dt == EXF_BF16) p.row_scale != nullptr ? run(yes, yes) : run(yes, no);
    else p.row_scale != nullptr ? run(no, yes) : run(no, no);
    return EXF_OK;
}

int launch_mx4_product(const Mx4Product& p, hipStream_t stream)
{
    const int64_t cols = (p.N + kMxTile - 1) / kMxTile, grid = (p.max_rows / kMxTile + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_mx4: too many tiles");
    hipLaunchKernelGGL(mx4_rows_kernel, dim3(static_cast<unsigned>(grid)), dim3(64), 0, stream, p, static_cast<int>(cols));
    return EXF_OK;
}

}  // namespace exf
