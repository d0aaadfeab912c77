// Launch interface of the experts' products (moe_grouped_product, its gradients, and operands in 4 bits).
#pragma once

#include "common.hpp"

namespace exf {

// out[rows of e, N] = rows[rows of e, K] * W_e (+ bias_e), a sorted row at a time:
//   forward    W_e [N,K] times the row:          weight [E_local,N,K], K = k, N = n
//   gradient   the row times W_e [K,N]:          weight [E_local,K,N], K = n, N = k
struct RowsProduct {
    const void* rows;         // [A,K]
    const int32_t* offsets;   // [E_local+1]
    const void* weight;
    const void* bias;         // [E_local,N] or null (forward)
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
// As RowsProduct, forward, of rows held by mx4_quantize; scales: [ceil(K/256), rows, 8].
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
int launch_exact_rows_product(const RowsProduct& p, bool gradient, hipStream_t stream);
int launch_exact_weight_gradient(const WeightGradient& p, hipStream_t stream);
int exact_weight_gradient_splits(int64_t A, int n, int k, int E_local);
// The sums of `splits` parts of n (and of m) values each, in order, in the type `dt`.
int launch_join_parts(const float* parts, int64_t n, void* out, const float* more, int64_t m, void* more_out, int splits, int dt, hipStream_t stream);
int launch_mx4_product(const Mx4Product& p, hipStream_t stream);  // result in fp32

// Bytes [a, a + n) and [b, b + m) overlap (nothing overlaps a null pointer).
inline bool overlap(const void* a, size_t n, const void* b, size_t m)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return a != nullptr && b != nullptr && p < q + m && q < p + n;
}

// ---- device side -------------------------------------------------------------------------
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
