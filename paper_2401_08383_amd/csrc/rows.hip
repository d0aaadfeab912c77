// moe_combine_topk, moe_combine_backward: the sorted rows of a token's assignments, summed by their weights, and the gradients of that.
// Streams over rows: 16 bytes of a row a lane.
#include "product.hpp"

namespace exf {

struct CombineCall {
    const uint4* y;              // [A, vecs]
    const int32_t* position;     // [T,k]
    const float* w;              // [T,k] or null (ones)
    uint4* out;                  // [T, vecs]
    int64_t T;
    int k, vecs, lanes;          // 16-byte pieces of a row; lanes of a token, a power of two
};
struct CombineGradient {
    const uint4* dout;           // [T, vecs]
    const uint4* y;              // [A, vecs] or null
    const int32_t* position;
    const float* w;              // [T,k] or null
    uint4* dy;                   // [A, vecs] or null
    float* dw;                   // [T,k] or null
    int64_t T;
    int k, vecs, lanes;
};

// A 16-byte piece in fp32.
template <bool BF16>
struct Piece {
    float v[BF16 ? 8 : 4];
};
template <bool BF16>
__device__ __forceinline__ Piece<BF16> unpack(uint4 t)
{
    const uint32_t u[4] = {t.x, t.y, t.z, t.w};
    Piece<BF16> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) r.v[2 * i] = __uint_as_float(u[i] << 16), r.v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        else r.v[i] = __uint_as_float(u[i]);
    }
    return r;
}
template <bool BF16>
__device__ __forceinline__ uint4 pack(const Piece<BF16>& r)
{
    if constexpr (BF16) return make_uint4(pack_bf16x2(r.v[0], r.v[1]), pack_bf16x2(r.v[2], r.v[3]), pack_bf16x2(r.v[4], r.v[5]), pack_bf16x2(r.v[6], r.v[7]));
    else return make_uint4(__float_as_uint(r.v[0]), __float_as_uint(r.v[1]), __float_as_uint(r.v[2]), __float_as_uint(r.v[3]));
}

constexpr int kRowsAhead = 8;  // rows of a token in flight

template <bool BF16>
__global__ __launch_bounds__(256) void combine_topk_kernel(const CombineCall p)
{
    constexpr int N = BF16 ? 8 : 4;
    const int64_t A = p.T * p.k, step = static_cast<int64_t>(gridDim.x) * (256 / p.lanes);
    const int in = threadIdx.x & (p.lanes - 1);
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * (256 / p.lanes) + threadIdx.x / p.lanes; t < p.T; t += step)
        for (int c = in; c < p.vecs; c += p.lanes) {
            Piece<BF16> sum;
#pragma unroll
            for (int i = 0; i < N; ++i) sum.v[i] = 0.0f;
            for (int j0 = 0; j0 < p.k; j0 += kRowsAhead) {
                uint4 v[kRowsAhead];
                float w[kRowsAhead];
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j) {
                    const int64_t a = t * p.k + j0 + j;
                    const int64_t s = j0 + j < p.k ? p.position[a] : -1;
                    const bool ok = s >= 0 && s < A;
                    v[j] = ok ? load_stream16(p.y + s * p.vecs + c) : make_uint4(0u, 0u, 0u, 0u);
                    w[j] = ok ? (p.w != nullptr ? p.w[a] : 1.0f) : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j) {
                    const Piece<BF16> r = unpack<BF16>(v[j]);
#pragma unroll
                    for (int i = 0; i < N; ++i) sum.v[i] = fmaf(w[j], r.v[i], sum.v[i]);
                }
            }
            store_stream16(p.out + t * p.vecs + c, pack<BF16>(sum));
        }
}

template <bool BF16>
__global__ __launch_bounds__(256) void combine_backward_kernel(const CombineGradient p)
{
    constexpr int N = BF16 ? 8 : 4;
    const int64_t A = p.T * p.k, step = static_cast<int64_t>(gridDim.x) * (256 / p.lanes);
    const int in = threadIdx.x & (p.lanes - 1);
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * (256 / p.lanes) + threadIdx.x / p.lanes; t < p.T; t += step)
        for (int j0 = 0; j0 < p.k; j0 += kRowsAhead) {
            int64_t at[kRowsAhead];
            float w[kRowsAhead], dot[kRowsAhead];
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j) {
                const int64_t a = t * p.k + j0 + j;
                const int64_t s = j0 + j < p.k ? p.position[a] : -1;
                at[j] = s < A ? s : -1;
                w[j] = at[j] >= 0 && p.w != nullptr ? p.w[a] : 1.0f;
                dot[j] = 0.0f;
            }
            for (int c = in; c < p.vecs; c += p.lanes) {
                const Piece<BF16> g = unpack<BF16>(p.dout[t * p.vecs + c]);
                uint4 v[kRowsAhead];
                if (p.dw != nullptr) {
#pragma unroll
                    for (int j = 0; j < kRowsAhead; ++j) v[j] = at[j] >= 0 ? load_stream16(p.y + at[j] * p.vecs + c) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int j = 0; j < kRowsAhead; ++j) {
                        const Piece<BF16> r = unpack<BF16>(v[j]);
                        if (at[j] >= 0)
#pragma unroll
                            for (int i = 0; i < N; ++i) dot[j] = fmaf(g.v[i], r.v[i], dot[j]);
                    }
                }
                if (p.dy != nullptr) {
#pragma unroll
                    for (int j = 0; j < kRowsAhead; ++j)
                        if (at[j] >= 0) {
                            Piece<BF16> r;
#pragma unroll
                            for (int i = 0; i < N; ++i) r.v[i] = w[j] * g.v[i];
                            store_stream16(p.dy + at[j] * p.vecs + c, pack<BF16>(r));
                        }
                }
            }
            if (p.dw != nullptr) {
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j) {
                    for (int off = p.lanes / 2; off > 0; off >>= 1) dot[j] += __shfl_xor(dot[j], off, kWave);
                    if (in == 0 && j0 + j < p.k) p.dw[t * p.k + j0 + j] = dot[j];
                }
            }
        }
}

static int check_rows(const char* fn, int64_t T, int d, int k, int dt)
{
    if (dt != EXF_F32 && dt != EXF_BF16) return fail(EXF_ERR_BAD_DTYPE, "%s: dt = %d", fn, dt);
    if (T < 0) return fail(EXF_ERR_BAD_SHAPE, "%s: T = %lld < 0", fn, static_cast<long long>(T));
    if (k < 1 || k > EXF_MAX_ROUTE_TOPK) return fail(EXF_ERR_BAD_SHAPE, "%s: k = %d outside [1,%d]", fn, k, EXF_MAX_ROUTE_TOPK);
    if (T >= (1ll << 31) / k) return fail(EXF_ERR_BAD_SHAPE, "%s: T*k must be below 2^31", fn);
    const int gran = dt == EXF_BF16 ? 8 : 4;
    if (d < gran || d % gran != 0 || d > EXF_MAX_PRODUCT_WIDTH)
        return fail(EXF_ERR_BAD_SHAPE, "%s: d = %d must be a positive multiple of %d, at most %d", fn, d, gran, EXF_MAX_PRODUCT_WIDTH);
    return EXF_OK;
}

static int lanes_for(int vecs)
{
    int lanes = 1;
    while (lanes < kWave && lanes < vecs) lanes *= 2;
    return lanes;
}
static unsigned rows_grid(int64_t T, int lanes)
{
    const int64_t blocks = (T * lanes + 255) / 256;
    return static_cast<unsigned>(blocks < 8 * kStreamWorkgroups ? blocks : 8 * kStreamWorkgroups);
}

}  // namespace exf

extern "C" int moe_combine_topk(const void* y_sorted, const int32_t* sorted_of_src, const float* topk_w, int64_t T, int d, int k, int dt, void* out,
                                void* stream)
{
    using namespace exf;
    const char* fn = "moe_combine_topk";
    if (int rc = check_rows(fn, T, d, k, dt)) return rc;
    if (T == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, y_sorted);
    EXF_CHECK_PTR(fn, sorted_of_src);
    EXF_CHECK_PTR(fn, out);
    EXF_CHECK_ALIGNED(fn, y_sorted);
    EXF_CHECK_ALIGNED(fn, out);
    const size_t row = static_cast<size_t>(d) * (dt == EXF_BF16 ? 2 : 4), o = T * row, slots = static_cast<size_t>(T) * k * 4;
    if (overlap(out, o, y_sorted, o * k) || overlap(out, o, sorted_of_src, slots) || overlap(out, o, topk_w, slots))
        return fail(EXF_ERR_BAD_SHAPE, "%s: the result must not overlap an input", fn);
    const int vecs = static_cast<int>(row / 16), lanes = lanes_for(vecs);
    const CombineCall p{static_cast<const uint4*>(y_sorted), sorted_of_src, topk_w, static_cast<uint4*>(out), T, k, vecs, lanes};
    const dim3 grid(rows_grid(T, lanes));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == EXF_BF16) hipLaunchKernelGGL(combine_topk_kernel<true>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(combine_topk_kernel<false>, grid, dim3(256), 0, s, p);
    return check_launch(fn);
}

extern "C" int moe_combine_backward(const void* dout, const void* y_sorted, const int32_t* sorted_of_src, const float* topk_w, int64_t T, int d, int k,
                                    int dt, void* dy_sorted, float* dtopk_w, void* stream)
{
    using namespace exf;
    const char* fn = "moe_combine_backward";
    if (int rc = check_rows(fn, T, d, k, dt)) return rc;
    if (T == 0 || (dy_sorted == nullptr && dtopk_w == nullptr)) return EXF_OK;
    EXF_CHECK_PTR(fn, dout);
    EXF_CHECK_PTR(fn, sorted_of_src);
    EXF_CHECK_ALIGNED(fn, dout);
    if (dtopk_w != nullptr) {
        EXF_CHECK_PTR(fn, y_sorted);
        EXF_CHECK_ALIGNED(fn, y_sorted);
    }
    if (dy_sorted != nullptr) {
        EXF_CHECK_PTR(fn, topk_w);
        EXF_CHECK_ALIGNED(fn, dy_sorted);
    }
    const size_t row = static_cast<size_t>(d) * (dt == EXF_BF16 ? 2 : 4), o = T * row, slots = static_cast<size_t>(T) * k * 4;
    const struct {
        const void* at;
        size_t bytes;
    } in[] = {{dout, o}, {y_sorted, o * k}, {sorted_of_src, slots}, {topk_w, slots}};
    for (const auto& i : in)
        if (overlap(dy_sorted, o * k, i.at, i.bytes) || overlap(dtopk_w, slots, i.at, i.bytes)) return fail(EXF_ERR_BAD_SHAPE, "%s: results must not overlap an input", fn);
    if (overlap(dy_sorted, o * k, dtopk_w, slots)) return fail(EXF_ERR_BAD_SHAPE, "%s: results must not overlap", fn);
    const int vecs = static_cast<int>(row / 16), lanes = lanes_for(vecs);
    const CombineGradient p{static_cast<const uint4*>(dout), static_cast<const uint4*>(y_sorted), sorted_of_src, topk_w, static_cast<uint4*>(dy_sorted), dtopk_w,
                            T, k, vecs, lanes};
    const dim3 grid(rows_grid(T, lanes));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == EXF_BF16) hipLaunchKernelGGL(combine_backward_kernel<true>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(combine_backward_kernel<false>, grid, dim3(256), 0, s, p);
    return check_launch(fn);
}
