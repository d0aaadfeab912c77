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

template <class F>
void pick_q4_group(int group, F run)
{
    if (group == 32) run(std::integral_constant<int, 32>());
    else if (group == 64) run(std::integral_constant<int, 64>());
    else run(std::integral_constant<int, 128>());
}

}  // namespace exf
