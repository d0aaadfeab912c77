// What the files of the 4-bit integers with group scales share.
#pragma once

#include <type_traits>

#include "product.hpp"

namespace exf {

// out[rows of e, N] = rows[rows of e, K] W_e^T (+ bias_e), W_e[n][u] = scale[e][n][u / group] (code[e][n][u] - zero[e][n][u / group]).
struct Q4Product {
    const void* rows;        // [A,K]
    const int32_t* offsets;  // [E_local+1]
    const uint8_t* weight;   // [E_local,N,K/2]
    const void* scale;       // [E_local,N,K/group], of the rows' type
    const uint8_t* zero;     // the same, bytes, or null (8)
    const void* bias;        // [E_local,N] or null
    void* out;               // [A,N]
    int max_rows, K, N, E_local;
};

inline int check_q4_group(const char* fn, int k, int group)
{
    if (group != 32 && group != 64 && group != 128) return fail(EXF_ERR_BAD_SHAPE, "%s: group = %d is none of 32, 64, 128", fn, group);
    if (k < group || k % group != 0) return fail(EXF_ERR_BAD_SHAPE, "%s: k = %d must be a positive multiple of the group, %d", fn, k, group);
    return EXF_OK;
}

// Zero points begin where those of an expert may: rows come in eights (bf16) or fours (fp32), a byte a group.  (The kernels load bytes, or words of four.)
inline int check_q4_zero(const char* fn, const uint8_t* zero, int dt)
{
    const unsigned by = dt == EXF_BF16 ? 8 : 4;
    if (reinterpret_cast<uintptr_t>(zero) % by != 0) return fail(EXF_ERR_MISALIGNED, "%s: the zero points are not %u-byte aligned", fn, by);
    return EXF_OK;
}

template <class F>
void pick_q4_group(int group, F run)
{
    if (group == 32) run(std::integral_constant<int, 32>());
    else if (group == 64) run(std::integral_constant<int, 64>());
    else run(std::integral_constant<int, 128>());
}

// bf16 products of many weights: operands staged through LDS (product_q4_stream.hip).
bool q4_streams(int64_t A, int n, int E_local);
int launch_q4_stream(const Q4Product& p, int group, hipStream_t stream);

// ---- device side -------------------------------------------------------------------------
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
// Eight codes as bf16 numbers 16 + code, in the order 0 4 1 5 2 6 3 7.  The constants come from registers: an instruction takes one literal, and
// "and, or" of two are one instruction.
struct CodeBits {
    uint32_t mask, sixteen;
};
__device__ __forceinline__ CodeBits code_bits()
{
    CodeBits b{0x00780078u, 0x41804180u};
    asm volatile("" : "+s"(b.mask), "+v"(b.sixteen));
    return b;
}
__device__ __forceinline__ bf16x8_t codes_bf16(uint32_t q, CodeBits b)
{
    return as_bf16x8(((q << 3) & b.mask) | b.sixteen, ((q >> 1) & b.mask) | b.sixteen, ((q >> 5) & b.mask) | b.sixteen, ((q >> 9) & b.mask) | b.sixteen);
}
__device__ __forceinline__ bf16x8_t ones_bf16() { return as_bf16x8(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u); }
// Eight bf16 numbers in that order.
__device__ __forceinline__ bf16x8_t in_code_order(uint4 x)
{
    auto low = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); };
    auto high = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); };
    return as_bf16x8(low(x.x, x.z), high(x.x, x.z), low(x.y, x.w), high(x.y, x.w));
}

// Memory at an address that is the same in every lane.
typedef const __attribute__((address_space(1))) uint8_t* global_bytes;
__device__ __forceinline__ global_bytes shared_place(const void* p)
{
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
    return reinterpret_cast<global_bytes>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ uint4 load_vector(global_bytes p)
{
    const u32x4_v v = *reinterpret_cast<const __attribute__((address_space(1))) u32x4_v*>(p);
    return uint4{v[0], v[1], v[2], v[3]};
}

// The value of each of the four quads, in all of them.
__device__ __forceinline__ void spread_quads(uint32_t v, uint32_t (&r)[4])
{
    r[0] = r[1] = r[2] = r[3] = v;
    turn_quads(r);
}

}  // namespace exf
