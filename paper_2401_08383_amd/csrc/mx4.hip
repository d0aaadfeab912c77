// mx4_quantize, mx4_dequantize: rows in blocks of 32 4-bit floating-point numbers with a common power of two.  Pure streams.
//
// A lane takes eight elements, four lanes a block, half a wavefront the 256 elements (a scale tile) of a row.  The largest magnitude's
// exponent bits are the scale (largest magnitude as an integer: infinities and NaN come out as 255 by themselves); the
// hardware's conversion divides by a power of two, rounds to nearest with ties to the even code and saturates, which is the
// definition, down to the scale 2^-127.
#include "product.hpp"

namespace exf {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;

constexpr int kScaleTile = 256;
constexpr int scale_tiles(int k) { return (k - 1) / kScaleTile + 1; }  // (k at least 1)
static_assert(scale_tiles(1) == 1 && scale_tiles(256) == 1 && scale_tiles(257) == 2 && scale_tiles(0x7fffffff) == 1 << 23, "any k there is");

template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const void* __restrict__ x, int64_t rows, int k, int tiles, uint32_t* __restrict__ q,
                                                           uint8_t* __restrict__ scale)
{
    const int lane = lane_id(), half = lane >> 5, chunk = lane & 31;
    const int64_t pairs = (rows + 1) / 2, items = pairs * tiles;  // an item: a tile of two rows
    const int64_t waves = static_cast<int64_t>(gridDim.x) * (blockDim.x / kWave);
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * (blockDim.x / kWave) + threadIdx.x / kWave; item < items; item += waves) {
        const int64_t row = item / tiles * 2 + half;
        const int tile = static_cast<int>(item % tiles), col = tile * kScaleTile + chunk * 8;
        const bool there = row < rows && col < k;
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0u;
        if (there) load_bits8<BF16>(static_cast<const uint8_t*>(x) + (row * k + col) * (BF16 ? 2 : 4), v);
        uint32_t largest = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) largest = max(largest, v[i] & 0x7fffffffu);
        largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 1, kWave)));
        largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), 2, kWave)));
        const uint32_t byte = scale_byte(largest);
        if (there) q[(row * k + col) / 8] = to_codes(v, byte);
        if (row < rows && (chunk & 3) == 0) scale[(tile * rows + row) * 8 + chunk / 4] = static_cast<uint8_t>(there ? byte : 0u);
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint32_t* __restrict__ q, const uint8_t* __restrict__ scale, int64_t rows, int k, int tiles,
                                                             void* __restrict__ out)
{
    const int lane = lane_id(), half = lane >> 5, chunk = lane & 31;
    const int64_t items = (rows + 1) / 2 * tiles, waves = static_cast<int64_t>(gridDim.x) * (blockDim.x / kWave);  // an item: a tile of two rows
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * (blockDim.x / kWave) + threadIdx.x / kWave; item < items; item += waves) {
        const int64_t row = item / tiles * 2 + half;
        const int tile = static_cast<int>(item % tiles), col = tile * kScaleTile + chunk * 8;
        if (row >= rows || col >= k) continue;
        const int64_t i = (row * k + col) / 8;
        const uint32_t byte = scale[(tile * rows + row) * 8 + chunk / 4], code = q[i];
        const float s = scale_value(byte == 255u ? 127u : byte);
        f32x2_t v[4];
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3);
        if (byte == 255u)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j][0] = v[j][1] = __uint_as_float(0x7fc00000u);
        if constexpr (BF16) {
            store_stream16(reinterpret_cast<uint4*>(out) + i, make_uint4(pack_bf16x2(v[0][0], v[0][1]), pack_bf16x2(v[1][0], v[1][1]),
                                                                         pack_bf16x2(v[2][0], v[2][1]), pack_bf16x2(v[3][0], v[3][1])));
        } else {
            auto bits = [](f32x2_t a, f32x2_t b) { return make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])); };
            store_stream16(reinterpret_cast<uint4*>(out) + 2 * i, bits(v[0], v[1]));
            store_stream16(reinterpret_cast<uint4*>(out) + 2 * i + 1, bits(v[2], v[3]));
        }
    }
}

static int check_mx4(const char* fn, const void* x, int64_t rows, int k, int dt, const uint8_t* q, const uint8_t* scale)
{
    if (dt != EXF_F32 && dt != EXF_BF16) return fail(EXF_ERR_BAD_DTYPE, "%s: dt = %d", fn, dt);
    if (k < EXF_MX4_BLOCK || k % EXF_MX4_BLOCK != 0) return fail(EXF_ERR_BAD_SHAPE, "%s: k = %d must be a positive multiple of %d", fn, k, EXF_MX4_BLOCK);
    if (rows < 0 || rows >= (1ll << 40) / k) return fail(EXF_ERR_BAD_SHAPE, "%s: rows = %lld outside [0, 2^40 / k)", fn, static_cast<long long>(rows));
    if (rows == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, x);
    EXF_CHECK_PTR(fn, q);
    EXF_CHECK_PTR(fn, scale);
    EXF_CHECK_ALIGNED(fn, x);
    EXF_CHECK_ALIGNED(fn, q);
    EXF_CHECK_ALIGNED(fn, scale);
    const size_t n = static_cast<size_t>(rows) * k, full = n * (dt == EXF_BF16 ? 2 : 4);
    if (overlap(x, full, q, n / 2) || overlap(x, full, scale, mx4_scale_bytes(rows, k)) || overlap(q, n / 2, scale, mx4_scale_bytes(rows, k)))
        return fail(EXF_ERR_BAD_SHAPE, "%s: the arrays must not overlap", fn);
    return EXF_OK;
}

}  // namespace exf

extern "C" size_t mx4_scale_bytes(int64_t rows, int k)
{
    if (rows < 0 || k < 1) return 0;
    return static_cast<size_t>(exf::scale_tiles(k)) * static_cast<size_t>(rows) * (exf::kScaleTile / EXF_MX4_BLOCK);
}

extern "C" int mx4_quantize(const void* x, int64_t rows, int k, int dt, uint8_t* q, uint8_t* scale, void* stream)
{
    using namespace exf;
    if (int rc = check_mx4("mx4_quantize", x, rows, k, dt, q, scale)) return rc;
    if (rows == 0) return EXF_OK;
    const int tiles = scale_tiles(k);
    const int64_t items = (rows + 1) / 2 * tiles;
    const unsigned grid = static_cast<unsigned>(items / 4 + 1 < 4 * kStreamWorkgroups ? items / 4 + 1 : 4 * kStreamWorkgroups);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == EXF_BF16) hipLaunchKernelGGL(mx4_quantize_kernel<true>, dim3(grid), dim3(256), 0, s, x, rows, k, tiles, reinterpret_cast<uint32_t*>(q), scale);
    else hipLaunchKernelGGL(mx4_quantize_kernel<false>, dim3(grid), dim3(256), 0, s, x, rows, k, tiles, reinterpret_cast<uint32_t*>(q), scale);
    return check_launch("mx4_quantize");
}

extern "C" int mx4_dequantize(const uint8_t* q, const uint8_t* scale, int64_t rows, int k, int dt, void* out, void* stream)
{
    using namespace exf;
    if (int rc = check_mx4("mx4_dequantize", out, rows, k, dt, q, scale)) return rc;
    if (rows == 0) return EXF_OK;
    const int tiles = scale_tiles(k);
    const int64_t items = (rows + 1) / 2 * tiles;
    const unsigned grid = static_cast<unsigned>(items / 4 + 1 < 4 * kStreamWorkgroups ? items / 4 + 1 : 4 * kStreamWorkgroups);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == EXF_BF16) hipLaunchKernelGGL(mx4_dequantize_kernel<true>, dim3(grid), dim3(256), 0, s, reinterpret_cast<const uint32_t*>(q), scale, rows, k, tiles, out);
    else hipLaunchKernelGGL(mx4_dequantize_kernel<false>, dim3(grid), dim3(256), 0, s, reinterpret_cast<const uint32_t*>(q), scale, rows, k, tiles, out);
    return check_launch("mx4_dequantize");
}
