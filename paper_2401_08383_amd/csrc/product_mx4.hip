// Grouped product of rows held in microscaled 4-bit floating point, on the block-scaled matrix instruction
// (v_mfma_scale_f32_16x16x128_f8f6f4): 16 x 16 outputs and 128 reduction elements at once, a lane with one block of 32 of a row, 16
// bytes, and that block's scale byte.
//
// A wavefront computes 64 x 64 outputs; operands come straight from memory.
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

int launch_mx4_product(const Mx4Product& p, hipStream_t stream)
{
    const int64_t cols = (p.N + kMxTile - 1) / kMxTile, grid = (p.max_rows / kMxTile + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_mx4: too many tiles");
    hipLaunchKernelGGL(mx4_rows_kernel, dim3(static_cast<unsigned>(grid)), dim3(64), 0, stream, p, static_cast<int>(cols));
    return EXF_OK;
}

}  // namespace exf
