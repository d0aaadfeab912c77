// Launch interface of the experts' products (moe_grouped_product, its gradients, and operands in 4 bits).
#pragma once

#include "common.hpp"

namespace exf {

// out[rows of e, N] = rows[rows of e, K] W_e^T (+ bias_e), weight [E_local,N,K], or in a rows' gradient rows W_e, weight [E_local,K,N].
struct ExactRows {
    const void* rows;         // [A,K]
    const int32_t* offsets;   // [E_local+1]
    const void* weight;
    const void* bias;         // [E_local,N] or null
    void* out;                // [A,N]
    int max_rows;             // A
    int K, N, E_local;
};
// out[e][N,K] = dy[rows of e, N]^T x[rows of e, K], the reduction over an expert's rows.
struct WeightGradient {
    const void* dy;
    const void* x;
    const int32_t* offsets;
    void* dw;
    void* db;                 // [E_local,N] or null
    void* workspace;
    int max_rows, N, K, E_local;
};
// out[rows of e, N] = rows[rows of e, K] W_e^T (+ bias_e) of operands held by mx4_quantize; scales: [ceil(K/256), rows, 8].
struct Mx4Product {
    const uint8_t* rows;
    const uint8_t* row_scale;
    const int32_t* offsets;
    const uint8_t* weight;
    const uint8_t* weight_scale;
    const void* bias;
    void* out;
    int max_rows, K, N, E_local;
};

// fp32 (product_exact.hip).
int launch_exact_product(const ExactRows& p, hipStream_t stream);
int launch_exact_rows_gradient(const ExactRows& p, hipStream_t stream);
int launch_exact_weight_gradient(const WeightGradient& p, hipStream_t stream);
int exact_weight_gradient_splits(int64_t A, int n, int k, int E_local);
// The sums of `splits` parts of n (and of m) values each, in order, in the type `dt`.
int launch_join_parts(const float* parts, int64_t n, void* out, const float* more, int64_t m, void* more_out, int splits, int dt, hipStream_t stream);
int launch_mx4_product(const Mx4Product& p, hipStream_t stream);  // result in fp32
// Small products: one launch, rows quantised where they are needed (rows of the result's type where row_scale is null).
bool mx4_product_is_small(int64_t A, int n, int k);
int launch_mx4_small(const Mx4Product& p, int dt, hipStream_t stream);

// Bytes [a, a + n) and [b, b + m) overlap (nothing overlaps a null pointer).
inline bool overlap(const void* a, size_t n, const void* b, size_t m)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return a != nullptr && b != nullptr && p < q + m && q < p + n;
}

// ---- device side -------------------------------------------------------------------------
// log2 X + 127 of a block of 4-bit numbers whose largest magnitude has these bits (see mx4.hip), and 2^(byte - 127).
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest)
{
    const uint32_t exponent = largest >> 23;
    return exponent == 255u ? 255u : max(exponent, 2u) - 2u;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte << 23); }
// Eight numbers, given by their bits, divided by the block's power of two and rounded to four bits each.
__device__ __forceinline__ uint32_t to_codes(const uint32_t (&v)[8], uint32_t byte)
{
    const float s = scale_value(byte == 255u ? 127u : byte);
    uint32_t code = 0u;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __uint_as_float(v[0]), __uint_as_float(v[1]), s, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __uint_as_float(v[2]), __uint_as_float(v[3]), s, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __uint_as_float(v[4]), __uint_as_float(v[5]), s, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __uint_as_float(v[6]), __uint_as_float(v[7]), s, 3);
    return byte == 255u ? 0u : code;
}
// Eight consecutive elements as the bits of fp32 numbers.
template <bool BF16>
__device__ __forceinline__ void load_bits8(const void* p, uint32_t (&v)[8])
{
    if constexpr (BF16) {
        const uint4 t = *static_cast<const uint4*>(p);
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = w[i] << 16, v[2 * i + 1] = w[i] & 0xffff0000u;
    } else {
        const uint4 a = static_cast<const uint4*>(p)[0], b = static_cast<const uint4*>(p)[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}

struct ExpertRows {  // rows [lo, hi) of expert `lane`
    int lo, hi;
};
// Clamped, so that no offsets lead past the arrays.
__device__ __forceinline__ ExpertRows expert_rows(const int32_t* __restrict__ offsets, int E_local, int max_rows)
{
    ExpertRows r{0, 0};
    const int lane = lane_id();
    if (lane < E_local) {
        r.lo = min(max(offsets[lane], 0), max_rows);
        r.hi = min(max(offsets[lane + 1], r.lo), max_rows);
    }
    return r;
}

}  // namespace exf
