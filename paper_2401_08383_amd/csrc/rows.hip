// moe_combine_topk, moe_combine_backward: the sorted rows of a token's assignments, summed by their weights, and the gradients of that; and the rows of
// moe_dispatch_topk's long lists.
// Streams over rows: 16 bytes of a row a lane.  HBM bounds them: 16384 tokens of 8 assignments, rows of 4 KiB, 605 MB in 105 us, 5.8 TB/s, the rate of a copy
// (a token a group of 64 lanes in the first form: 139); gradients of 8192 x 8 571 MB in 107, 5.3 TB/s (141).  Short calls: 4.0 and 4.4 us for 333 x 6 rows of 4 KiB and
// 129 x 3 of 2 KiB, a launch and two loads that follow one another.
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

// Rows of more than 32 pieces: a token a wavefront, or `waves` (1, 2, 4) of them a token, which share its columns: a row is read at one time.  Its positions and
// weights are fetched by a lane each and handed out on the scalar path, those of the wavefront's next token while this one's rows travel, and U pieces a lane of
// every row are in flight.
constexpr int kRowsPieces = 2;

struct Assigned {  // what lane j has of slot j
    int at;
    float w;
};
__device__ __forceinline__ Assigned assigned(const int32_t* position, const float* w, int64_t t, int64_t T, int k, int64_t A, int lane)
{
    Assigned r{-1, 1.0f};
    if (t < T && lane < k) {
        const int64_t s = position[t * k + lane];
        r.at = s < A ? static_cast<int>(s) : -1;
        if (w != nullptr) r.w = w[t * k + lane];
    }
    return r;
}

template <bool BF16>
__global__ __launch_bounds__(256) void combine_wave_kernel(const CombineCall p, int waves)
{
    constexpr int N = BF16 ? 8 : 4, U = kRowsPieces;
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), share = wave & (waves - 1), tokens = 4 / waves;
    const int64_t A = p.T * p.k, step = static_cast<int64_t>(gridDim.x) * tokens;
    int64_t t = static_cast<int64_t>(blockIdx.x) * tokens + wave / waves;
    Assigned next = assigned(p.position, p.w, t, p.T, p.k, A, lane);
    for (; t < p.T; t += step) {
        const Assigned mine = next;
        next = assigned(p.position, p.w, t + step, p.T, p.k, A, lane);
        for (int c0 = share * kWave * U + lane; c0 < p.vecs; c0 += waves * kWave * U) {
            Piece<BF16> sum[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[u].v[i] = 0.0f;
            for (int j0 = 0; j0 < p.k; j0 += kRowsAhead) {
                uint4 v[kRowsAhead][U];
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j) {
                    const int s = wave_read_lane(mine.at, j0 + j);  // (-1 past the last slot)
                    const uint4* row = p.y + static_cast<int64_t>(max(s, 0)) * p.vecs;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        v[j][u] = make_uint4(0u, 0u, 0u, 0u);
                        if (s >= 0 && c0 + u * kWave < p.vecs) v[j][u] = load_stream16(row + (c0 + u * kWave));
                    }
                }
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j) {
                    const bool there = wave_read_lane(mine.at, j0 + j) >= 0;
                    const float w = there ? __int_as_float(wave_read_lane(__float_as_int(mine.w), j0 + j)) : 0.0f;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const Piece<BF16> r = unpack<BF16>(v[j][u]);
#pragma unroll
                        for (int i = 0; i < N; ++i) sum[u].v[i] = fmaf(w, r.v[i], sum[u].v[i]);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u * kWave < p.vecs) store_stream16(p.out + t * p.vecs + c0 + u * kWave, pack<BF16>(sum[u]));
        }
    }
}

// Gradients: the wavefronts of a token join their sums through LDS, in order.
template <bool BF16>
__global__ __launch_bounds__(256) void combine_backward_wave_kernel(const CombineGradient p, int waves)
{
    __shared__ float part[4][kRowsAhead];
    constexpr int N = BF16 ? 8 : 4;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), share = wave & (waves - 1);
    const int64_t A = p.T * p.k, tokens = 4 / waves, step = static_cast<int64_t>(gridDim.x) * tokens;
    int64_t t = static_cast<int64_t>(blockIdx.x) * tokens + wave / waves;
    Assigned next = assigned(p.position, p.w, t, p.T, p.k, A, lane);
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens; t0 < p.T; t0 += step, t += step) {  // (the same number of times for all wavefronts)
        const Assigned mine = next;
        next = assigned(p.position, p.w, t + step, p.T, p.k, A, lane);
        const int vecs = t < p.T ? p.vecs : 0;
        for (int j0 = 0; j0 < p.k; j0 += kRowsAhead) {
            float dot[kRowsAhead];
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j) dot[j] = 0.0f;
            for (int c = share * kWave + lane; c < vecs; c += waves * kWave) {
                const uint4 g4 = p.dout[t * p.vecs + c];
                uint4 v[kRowsAhead];
                if (p.dw != nullptr) {
#pragma unroll
                    for (int j = 0; j < kRowsAhead; ++j) {
                        const int s = wave_read_lane(mine.at, j0 + j);
                        v[j] = make_uint4(0u, 0u, 0u, 0u);
                        if (s >= 0) v[j] = load_stream16(p.y + static_cast<int64_t>(s) * p.vecs + c);
                    }
                }
                const Piece<BF16> g = unpack<BF16>(g4);
                if (p.dy != nullptr) {
#pragma unroll
                    for (int j = 0; j < kRowsAhead; ++j) {
                        const int s = wave_read_lane(mine.at, j0 + j);
                        if (s < 0) continue;
                        const float w = __int_as_float(wave_read_lane(__float_as_int(mine.w), j0 + j));
                        Piece<BF16> r;
#pragma unroll
                        for (int i = 0; i < N; ++i) r.v[i] = w * g.v[i];
                        store_stream16(p.dy + static_cast<int64_t>(s) * p.vecs + c, pack<BF16>(r));
                    }
                }
                if (p.dw != nullptr) {
#pragma unroll
                    for (int j = 0; j < kRowsAhead; ++j) {
                        if (wave_read_lane(mine.at, j0 + j) < 0) continue;
                        const Piece<BF16> r = unpack<BF16>(v[j]);
#pragma unroll
                        for (int i = 0; i < N; ++i) dot[j] = fmaf(g.v[i], r.v[i], dot[j]);
                    }
                }
            }
            if (p.dw == nullptr) continue;
            float all = 0.0f;
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j) {
                const float sum = wave_sum(dot[j]);
                all = lane == j ? sum : all;
            }
            if (waves > 1) {
                if (lane < kRowsAhead) part[wave][lane] = all;
                __syncthreads();
                if (lane < kRowsAhead) {
                    all = part[wave - share][lane] + part[wave - share + 1][lane];
                    if (waves == 4) all += part[2][lane] + part[3][lane];
                }
                __syncthreads();
            }
            if (t < p.T && share == 0 && lane < kRowsAhead && j0 + lane < p.k) p.dw[t * p.k + j0 + lane] = all;
        }
    }
}

// Rows of moe_dispatch_topk: a token's row is read once and written to the places of its assignments.  HBM bounds it, and how writes of a row each fill its pages: 16384
// tokens of 8, rows of 4 KiB, 604 MB 133 us with the list's positions (13), of which 119 for the rows, 5.1 TB/s; two wavefronts a token with streaming stores 138, four 131, a wavefront with
// these 136; rows in the order of their places, each read for itself, 166 (of the dispatch of one or two assignments 188).  8192 tokens 58, 73, 71, 72, 86 and 90.
struct SpreadCall {
    const uint4* x;           // [T, vecs]
    const int32_t* position;  // [T,k]
    uint4* out;               // [A, vecs]
    int64_t T;
    int k, vecs, lanes;
};
__global__ __launch_bounds__(256) void spread_kernel(const SpreadCall p)
{
    const int64_t A = p.T * p.k, step = static_cast<int64_t>(gridDim.x) * (256 / p.lanes);
    const int in = threadIdx.x & (p.lanes - 1);
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * (256 / p.lanes) + threadIdx.x / p.lanes; t < p.T; t += step)
        for (int c = in; c < p.vecs; c += p.lanes) {
            const uint4 v = p.x[t * p.vecs + c];
            for (int j0 = 0; j0 < p.k; j0 += kRowsAhead) {
                int64_t at[kRowsAhead];
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j) at[j] = j0 + j < p.k ? p.position[t * p.k + j0 + j] : -1;
#pragma unroll
                for (int j = 0; j < kRowsAhead; ++j)
                    if (at[j] >= 0 && at[j] < A) store_stream16(p.out + at[j] * p.vecs + c, v);
            }
        }
}
// A token a wavefront, all of a row of up to 4 KiB in flight.  Not with streaming stores: who reads the rows next finds a part of them behind the L2 (8192 tokens, buffers that change from
// call to call: 70 us with either, with moe_combine behind it 99 and 122 for both).
__global__ __launch_bounds__(256) void spread_wave_kernel(const SpreadCall p)
{
    constexpr int U = 4;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t A = p.T * p.k, step = static_cast<int64_t>(gridDim.x) * 4;
    int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    Assigned next = assigned(p.position, nullptr, t, p.T, p.k, A, lane);
    for (; t < p.T; t += step) {
        const Assigned mine = next;
        next = assigned(p.position, nullptr, t + step, p.T, p.k, A, lane);
        for (int c0 = lane; c0 < p.vecs; c0 += kWave * U) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u * kWave < p.vecs) v[u] = load_stream16(p.x + t * p.vecs + c0 + u * kWave);
            for (int j = 0; j < p.k; ++j) {
                const int s = wave_read_lane(mine.at, j);
                if (s < 0) continue;
                uint4* row = p.out + static_cast<int64_t>(s) * p.vecs;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c0 + u * kWave < p.vecs) row[c0 + u * kWave] = v[u];
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

void launch_spread(const void* x, const int32_t* position, int64_t T, int k, int vecs, void* out, hipStream_t stream)
{
    // Rows of 1 KiB and less, the list's positions included: 512 bytes of 32768 x 8 43 us with lanes a token, 50 with a wavefront; rows of 2 KiB of 32768 x 4 65 and 67, of 4 KiB of
    // 8192 x 8 84 and 58.
    const int lanes = lanes_for(vecs);
    const SpreadCall p{static_cast<const uint4*>(x), position, static_cast<uint4*>(out), T, k, vecs, lanes};
    if (vecs > kWave) hipLaunchKernelGGL(spread_wave_kernel, dim3(rows_grid(T, kWave)), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(spread_kernel, dim3(rows_grid(T, lanes)), dim3(256), 0, stream, p);
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
    // Rows of 4 KiB of 16384 x 8 assignments 105 us with one wavefront a token and with two, of 8192 x 8 56 and 52, of 8 KiB of 8192 x 2 42 and 37, of 1 KiB of 65536 x 4
    // 64 and 82; of 4 KiB of 333 x 6 6.1, 4.9 and with four 4.0.
    const int waves = vecs <= 2 * kWave ? 1 : (T < 1024 ? 4 : 2);
    if (lanes == kWave && dt == EXF_BF16) hipLaunchKernelGGL(combine_wave_kernel<true>, dim3(rows_grid(T, lanes * waves)), dim3(256), 0, s, p, waves);
    else if (lanes == kWave) hipLaunchKernelGGL(combine_wave_kernel<false>, dim3(rows_grid(T, lanes * waves)), dim3(256), 0, s, p, waves);
    else if (dt == EXF_BF16) hipLaunchKernelGGL(combine_topk_kernel<true>, grid, dim3(256), 0, s, p);
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
    // Rows of 4 KiB of 8192 x 8 assignments 119 us with one wavefront a token, 109 with two, 104 with four; of 8 KiB of 8192 x 2 67, 61 and 56; of 1 KiB of 65536 x 4 103, 111
    // and 155; of 2 KiB of 129 x 3 6.2, 5.1 and 4.2.
    const int waves = vecs > 2 * kWave ? 4 : (vecs > kWave ? 2 : 1);
    if (lanes == kWave && dt == EXF_BF16) hipLaunchKernelGGL(combine_backward_wave_kernel<true>, dim3(rows_grid(T, lanes * waves)), dim3(256), 0, s, p, waves);
    else if (lanes == kWave) hipLaunchKernelGGL(combine_backward_wave_kernel<false>, dim3(rows_grid(T, lanes * waves)), dim3(256), 0, s, p, waves);
    else if (dt == EXF_BF16) hipLaunchKernelGGL(combine_backward_kernel<true>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(combine_backward_kernel<false>, grid, dim3(256), 0, s, p);
    return check_launch(fn);
}
