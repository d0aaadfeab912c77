// The experts' products in fp32 arithmetic on the matrix cores: fp32 operands.
//
// A workgroup of four wavefronts computes 64 x 64 outputs, a wavefront 32 x 32 in 16x16 accumulators (v_mfma_f32_16x16x4_f32).
// Operands go through registers into LDS, the next stage of 32 reduction elements on its way while one is multiplied.  An
// operand whose reduction lies along memory is kept [row][reduction] and fetched four elements at a time (a lane's four
// elements meet the other operand's in four instructions; which four a step sums does not matter as long as both operands
// agree); one whose reduction lies across memory is kept as it comes, [reduction][row].
//   Two sets of accumulators take turns every 16 elements: the sum of a long reduction then has half as many roundings in a row.
#include "product.hpp"

namespace exf {

constexpr int kExactTile = 64, kExactDepth = 32;

__device__ __forceinline__ f32x4_t load4(const float* p) { return *reinterpret_cast<const f32x4_t*>(p); }

// One operand of a tile: 64 rows (output rows or columns) of the reduction [0, depth).
//   ACROSS false: element (row, r) at base[row * ld + r];  true: at base[r * ld + row].
template <bool ACROSS>
struct ExactOperand {
    static constexpr int STRIDE = ACROSS ? kExactTile + 4 : kExactDepth + 4;
    static constexpr int FLOATS = ACROSS ? kExactDepth * STRIDE : kExactTile * STRIDE;
    const float* base;
    int64_t ld;
    int rows, depth;
    f32x4_t v[2];

    __device__ __forceinline__ void load(int r0)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = threadIdx.x + i * 256;
            const int row = ACROSS ? t % 16 * 4 : t / 8, r = r0 + (ACROSS ? t / 16 : t % 8 * 4);
            v[i] = row < rows && r < depth ? load4(base + (ACROSS ? static_cast<int64_t>(r) * ld + row : static_cast<int64_t>(row) * ld + r)) : f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void store(float* lds) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = threadIdx.x + i * 256;
            *reinterpret_cast<f32x4_t*>(lds + (ACROSS ? t / 16 * STRIDE + t % 16 * 4 : t / 8 * STRIDE + t % 8 * 4)) = v[i];
        }
    }
    // elements r .. r+3 of a row
    __device__ __forceinline__ f32x4_t fetch(const float* lds, int row, int r) const
    {
        if constexpr (!ACROSS) return *reinterpret_cast<const f32x4_t*>(lds + row * STRIDE + r);
        return f32x4_t{lds[r * STRIDE + row], lds[(r + 1) * STRIDE + row], lds[(r + 2) * STRIDE + row], lds[(r + 3) * STRIDE + row]};
    }
};

// D[row][col] = sum_r a(row, r) w(col, r) + bias[col], written where row < a.rows and col < w.rows; sums[row] = sum_r a(row, r) where wanted
// (a across).
template <bool A_ACROSS, bool W_ACROSS>
__device__ __forceinline__ void exact_tile(ExactOperand<A_ACROSS> a, ExactOperand<W_ACROSS> w, const float* bias, float* out, int64_t ldo, float* sums = nullptr)
{
    typedef ExactOperand<A_ACROSS> OA;
    typedef ExactOperand<W_ACROSS> OW;
    __shared__ __attribute__((aligned(16))) float lds[OA::FLOATS + OW::FLOATS];
    float *la = lds, *lw = lds + OA::FLOATS;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int row0 = wave / 2 * 32, col0 = wave % 2 * 32, in16 = lane & 15, quad = lane >> 4;
    f32x4_t acc[2][2][2];
    float sum = 0.0f;  // of row `lane`, a quarter of each stage
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[s][i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    a.load(0);
    w.load(0);
    for (int r0 = 0; r0 < a.depth; r0 += kExactDepth) {
        a.store(la);
        w.store(lw);
        __syncthreads();
        if (r0 + kExactDepth < a.depth) {
            a.load(r0 + kExactDepth);
            w.load(r0 + kExactDepth);
        }
        if (A_ACROSS && sums != nullptr)
#pragma unroll
            for (int r = 0; r < kExactDepth / 4; ++r) sum += la[(wave * (kExactDepth / 4) + r) * OA::STRIDE + lane];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f32x4_t fa[2], fw[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fa[i] = a.fetch(la, row0 + i * 16 + in16, s * 16 + quad * 4);
                fw[i] = w.fetch(lw, col0 + i * 16 + in16, s * 16 + quad * 4);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[s][i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[j][q], fa[i][q], acc[s][i][j], 0, 0, 0);
        }
        __syncthreads();
    }
    if (A_ACROSS && sums != nullptr) {
        lds[threadIdx.x] = sum;
        __syncthreads();
        if (wave == 0 && lane < a.rows) sums[lane] = (lds[lane] + lds[kWave + lane]) + (lds[2 * kWave + lane] + lds[3 * kWave + lane]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = row0 + i * 16 + in16, col = col0 + j * 16 + quad * 4;
            if (row >= a.rows || col >= w.rows) continue;
            f32x4_t v = acc[0][i][j] + acc[1][i][j];
            if (bias != nullptr) v += load4(bias + col);
            *reinterpret_cast<f32x4_t*>(out + static_cast<int64_t>(row) * ldo + col) = v;
        }
}

template <bool GRADIENT>
__global__ __launch_bounds__(256) void exact_rows_kernel(const RowsProduct p, int col_tiles)
{
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + kExactTile - 1) / kExactTile;
    const int upto = wave_inclusive_scan(tiles);
    const int row_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(col_tiles)), col_tile = static_cast<int>(blockIdx.x % static_cast<unsigned>(col_tiles));
    const unsigned long long owner = __ballot(row_tile < upto);
    if (owner == 0ull) return;
    const int e = __builtin_ctzll(owner);
    const int hi = wave_read_lane(range.hi, e);
    const int row = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * kExactTile;
    const int col = col_tile * kExactTile;
    const int64_t K = p.K, N = p.N;
    const float* weight = static_cast<const float*>(p.weight) + e * N * K;
    const ExactOperand<false> a{static_cast<const float*>(p.rows) + row * K, K, min(kExactTile, hi - row), p.K, {}};
    const ExactOperand<GRADIENT> w{GRADIENT ? weight + col : weight + col * K, GRADIENT ? N : K, min(kExactTile, p.N - col), p.K, {}};
    exact_tile(a, w, p.bias != nullptr ? static_cast<const float*>(p.bias) + e * N + col : nullptr, static_cast<float*>(p.out) + row * N + col, N);
}

// Parts of the reduction (blockIdx.y) go to [part][E_local][N,K] and sums to [part][E_local][N].
__global__ __launch_bounds__(256) void exact_weight_kernel(const WeightGradient p, int row_tiles, int col_tiles)
{
    const unsigned per_expert = static_cast<unsigned>(row_tiles) * static_cast<unsigned>(col_tiles);
    const int e = static_cast<int>(blockIdx.x / per_expert);
    const unsigned t = blockIdx.x % per_expert;
    const int row = static_cast<int>(t / static_cast<unsigned>(col_tiles)) * kExactTile, col = static_cast<int>(t % static_cast<unsigned>(col_tiles)) * kExactTile;
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int lo = wave_read_lane(range.lo, e), all = wave_read_lane(range.hi, e) - lo;
    const int stages = (all + kExactDepth - 1) / kExactDepth;
    const int first = static_cast<int>(static_cast<int64_t>(stages) * blockIdx.y / gridDim.y) * kExactDepth;
    const int n = max(min(all, static_cast<int>(static_cast<int64_t>(stages) * (blockIdx.y + 1) / gridDim.y) * kExactDepth) - first, 0);
    const int64_t N = p.N, K = p.K, begin = lo + first, at = static_cast<int64_t>(blockIdx.y) * p.E_local + e;
    const ExactOperand<true> a{static_cast<const float*>(p.dy) + begin * N + row, N, min(kExactTile, p.N - row), n, {}};
    const ExactOperand<true> w{static_cast<const float*>(p.x) + begin * K + col, K, min(kExactTile, p.K - col), n, {}};
    exact_tile(a, w, nullptr, static_cast<float*>(p.dw) + (at * N + row) * K + col, K, p.db != nullptr && col == 0 ? static_cast<float*>(p.db) + at * N + row : nullptr);
}

template <typename TO>
__global__ __launch_bounds__(256) void join_parts_kernel(const float* __restrict__ parts, int64_t quads, TO* __restrict__ out, const float* __restrict__ more,
                                                         int64_t more_quads, TO* __restrict__ more_out, int splits)
{
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < quads + more_quads; i += static_cast<int64_t>(gridDim.x) * 256) {
        const bool first = i < quads;
        const int64_t at = first ? i : i - quads, each = first ? quads : more_quads;
        const f32x4_t* from = reinterpret_cast<const f32x4_t*>(first ? parts : more) + at;
        f32x4_t sum = from[0];
        for (int s = 1; s < splits; ++s) sum += from[s * each];
        TO* to = (first ? out : more_out) + at * 4;
        if constexpr (sizeof(TO) == 4) *reinterpret_cast<f32x4_t*>(to) = sum;
        else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3]));
    }
}
int launch_join_parts(const float* parts, int64_t n, void* out, const float* more, int64_t m, void* more_out, int splits, int dt, hipStream_t stream)
{
    const int64_t blocks = ((n + m) / 4 + 255) / 256;
    const dim3 grid(static_cast<unsigned>(blocks < 4 * kStreamWorkgroups ? blocks : 4 * kStreamWorkgroups));
    if (dt == EXF_F32) hipLaunchKernelGGL(join_parts_kernel<float>, grid, dim3(256), 0, stream, parts, n / 4, static_cast<float*>(out), more, m / 4, static_cast<float*>(more_out), splits);
    else hipLaunchKernelGGL(join_parts_kernel<bf16_t>, grid, dim3(256), 0, stream, parts, n / 4, static_cast<bf16_t*>(out), more, m / 4, static_cast<bf16_t*>(more_out), splits);
    return EXF_OK;
}

static int64_t tiles_of(int64_t n) { return (n + kExactTile - 1) / kExactTile; }

int launch_exact_rows_product(const RowsProduct& p, bool gradient, hipStream_t stream)
{
    const int64_t cols = tiles_of(p.N), grid = (p.max_rows / kExactTile + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product: too many tiles");
    if (gradient) hipLaunchKernelGGL(exact_rows_kernel<true>, dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p, static_cast<int>(cols));
    else hipLaunchKernelGGL(exact_rows_kernel<false>, dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p, static_cast<int>(cols));
    return EXF_OK;
}
// Parts of at least 256 rows until two workgroups a compute unit have one.
int exact_weight_gradient_splits(int64_t A, int n, int k, int E_local)
{
    const int64_t wanted = 512 / (E_local * tiles_of(n) * tiles_of(k)), most = A / (256 * E_local);
    const int64_t s = wanted < most ? wanted : most;
    return static_cast<int>(s < 2 ? 1 : (s > 16 ? 16 : s));
}
int launch_exact_weight_gradient(const WeightGradient& g, hipStream_t stream)
{
    const int64_t rows = tiles_of(g.N), cols = tiles_of(g.K), grid = g.E_local * rows * cols, each = static_cast<int64_t>(g.E_local) * g.N * g.K;
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_dw: too many tiles");
    const int splits = exact_weight_gradient_splits(g.max_rows, g.N, g.K, g.E_local);
    float* parts = static_cast<float*>(g.workspace);
    WeightGradient p = g;
    if (splits > 1) {
        p.dw = parts;
        if (p.db != nullptr) p.db = parts + splits * each;
    }
    hipLaunchKernelGGL(exact_weight_kernel, dim3(static_cast<unsigned>(grid), static_cast<unsigned>(splits)), dim3(256), 0, stream, p, static_cast<int>(rows), static_cast<int>(cols));
    if (splits == 1) return EXF_OK;
    return launch_join_parts(parts, each, g.dw, parts + splits * each, g.db != nullptr ? static_cast<int64_t>(g.E_local) * g.N : 0, g.db, splits, EXF_F32, stream);
}

}  // namespace exf
