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

// D[row][col] = sum_r a(row, r) w(col, r), written where row < a.rows and col < w.rows; sums[row] = sum_r a(row, r) where wanted
// (a across); bias[col] is added where there is one.
template <bool A_ACROSS, bool W_ACROSS>
__device__ __forceinline__ void exact_tile(ExactOperand<A_ACROSS> a, ExactOperand<W_ACROSS> w, float* out, int64_t ldo, float* sums, const float* bias)
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
            const f32x4_t sum = acc[0][i][j] + acc[1][i][j];
            *reinterpret_cast<f32x4_t*>(out + static_cast<int64_t>(row) * ldo + col) = bias != nullptr ? sum + load4(bias + col) : sum;
        }
}

// ---- small problems: 16 (products, rows' gradients) or 32 (weights' gradient) x 64 outputs a workgroup, whose four wavefronts share the reduction
// (16 elements each in turn) and join their sums through LDS.  Operands come straight from memory into the registers that the matrix
// instructions read, kAhead turns early.
//   An operand across the reduction is loaded as it lies: a lane takes 16 bytes of a reduction element, four columns, and each of the four
// is the operand of a matrix instruction of its own, whose 16 columns are then four apart.  (Loads of 4 bytes for 16 adjacent columns are
// four times as many: gradient of 777 rows, 5 experts of 520 x 264 9.6 us with them, 8.9 without; with 16 rows a tile 7.3 to 8.1.)
// Loads past the end deliver zeros (see product_tiles.hpp).
//   A 16 x 16 x 4 product in fp32 takes 32 cycles, and few tiles are as fast as one of them: products and rows' gradients, whose
// experts often have few rows, take 16.
constexpr int kSmallCols = 64, kAhead = 3;
constexpr int small_rows(bool across) { return across ? 32 : 16; }
constexpr int kSmallStride = kSmallCols + 4;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const float* base, int64_t floats)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, static_cast<int>(floats * 4), 0x00020000);
}

// A_ACROSS: a's element (row, r) at a[r * lda + row], otherwise a[row * lda + r]; W_ACROSS and w's element (col, r) alike.
template <bool A_ACROSS, bool W_ACROSS>
__device__ __forceinline__ void small_tile(const float* a, int64_t lda, int rows, const float* w, int64_t ldw, int cols, int depth, float* out, int64_t ldo, float* sums,
                                           const float* bias)
{
    constexpr int ROWS = small_rows(A_ACROSS), R = ROWS / 16;  // row groups
    __shared__ __attribute__((aligned(16))) float part[4][ROWS * kSmallStride];
    __shared__ float part_sum[4][ROWS];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), in16 = lane & 15, quad = lane >> 4;
    // byte distances from the first of the 16 reduction elements
    int off_w[4], off_a[A_ACROSS ? 4 : R];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        off_w[q] = static_cast<int>((W_ACROSS ? (quad * 4 + q) * ldw + min(in16 * 4, cols - 4) : min(q * 16 + in16, cols - 1) * ldw + quad * 4) * 4);
        if constexpr (A_ACROSS) off_a[q] = static_cast<int>(((quad * 4 + q) * lda + min(in16 * 2, rows - 2)) * 4);
    }
    if constexpr (!A_ACROSS)
#pragma unroll
        for (int i = 0; i < R; ++i) off_a[i] = static_cast<int>((min(i * 16 + in16, rows - 1) * lda + quad * 4) * 4);
    f32x4_t acc[R][4];
    f32x4_t fw[kAhead][4];   // across: [reduction element] of a lane's four columns; along: [16 columns] of its four reduction elements
    float fa[kAhead][R][4];  // [row group][reduction element]
    float sum[R] = {};
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto load = [&](int turn, int s) {
        const int begin = (turn * 4 + wave) * 16, left = depth - begin, last = min(left, 16) - 1;
        const auto from_w = W_ACROSS ? buffer_of(w + begin * ldw, left > 0 ? last * ldw + cols : 0) : buffer_of(w + begin, left > 0 ? (cols - 1) * ldw + left : 0);
#pragma unroll
        for (int q = 0; q < 4; ++q)  // (a depth along memory is a multiple of four: all four or none)
            fw[s][q] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from_w, W_ACROSS || quad * 4 < left ? off_w[q] : -16, 0, 0));
        if constexpr (A_ACROSS) {
            const auto from_a = buffer_of(a + begin * lda, left > 0 ? last * lda + rows : 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const auto v = __builtin_amdgcn_raw_buffer_load_b64(from_a, off_a[q], 0, 0);
                fa[s][0][q] = __uint_as_float(v[0]);
                fa[s][1][q] = __uint_as_float(v[1]);
            }
        } else {
            const auto from_a = buffer_of(a + begin, left > 0 ? (rows - 1) * lda + left : 0);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const f32x4_t v = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from_a, quad * 4 < left ? off_a[i] : -16, 0, 0));
#pragma unroll
                for (int q = 0; q < 4; ++q) fa[s][i][q] = v[q];
            }
        }
    };
    const int turns = depth > wave * 16 ? (depth - wave * 16 + 63) / 64 : 0;
    if (turns > 0) {
#pragma unroll
        for (int s = 0; s < kAhead; ++s) load(s, s);
        for (int t = 0; t < turns; t += kAhead) {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(W_ACROSS ? fw[s][q][j] : fw[s][j][q], fa[s][i][q], acc[i][j], 0, 0, 0);
                if (A_ACROSS && sums != nullptr)
#pragma unroll
                    for (int i = 0; i < R; ++i) sum[i] += (fa[s][i][0] + fa[s][i][1]) + (fa[s][i][2] + fa[s][i][3]);
                load(t + s + kAhead, s);
            }
        }
    }
    // a lane holds in acc[i][j][v], of row group i, column 16 quad + 4 v + j of a w across, 16 j + 4 quad + v of one along
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = A_ACROSS ? in16 * 2 + i : i * 16 + in16;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            *reinterpret_cast<f32x4_t*>(&part[wave][row * kSmallStride + (W_ACROSS ? quad * 16 + v * 4 : v * 16 + quad * 4)]) =
                W_ACROSS ? f32x4_t{acc[i][0][v], acc[i][1][v], acc[i][2][v], acc[i][3][v]} : acc[i][v];
        if (A_ACROSS && sums != nullptr) {
            sum[i] = butterfly_add<16>(butterfly_add<32>(sum[i]));
            if (quad == 0) part_sum[wave][row] = sum[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < R; ++h) {
        const int r = threadIdx.x / 16 + h * 16, c = threadIdx.x % 16 * 4, at = r * kSmallStride + c;
        auto of = [&](int wv) { return *reinterpret_cast<const f32x4_t*>(&part[wv][at]); };
        if (r >= rows || c >= cols) continue;
        const f32x4_t sum = (of(0) + of(1)) + (of(2) + of(3));
        *reinterpret_cast<f32x4_t*>(out + r * ldo + c) = bias != nullptr ? sum + load4(bias + c) : sum;
    }
    if (A_ACROSS && sums != nullptr && static_cast<int>(threadIdx.x) < min(ROWS, rows))
        sums[threadIdx.x] = (part_sum[0][threadIdx.x] + part_sum[1][threadIdx.x]) + (part_sum[2][threadIdx.x] + part_sum[3][threadIdx.x]);
}

// W_ACROSS: rows' gradients; otherwise products.
template <bool SMALL, bool W_ACROSS>
__global__ __launch_bounds__(256) void exact_rows_kernel(const ExactRows p, int col_tiles)
{
    constexpr int ROWS = SMALL ? small_rows(false) : kExactTile, COLS = SMALL ? kSmallCols : kExactTile;
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + ROWS - 1) / ROWS;
    const int upto = wave_inclusive_scan(tiles);
    const int row_tile = static_cast<int>(blockIdx.x / static_cast<unsigned>(col_tiles)), col_tile = static_cast<int>(blockIdx.x % static_cast<unsigned>(col_tiles));
    const unsigned long long owner = __ballot(row_tile < upto);
    if (owner == 0ull) return;
    const int e = __builtin_ctzll(owner);
    const int hi = wave_read_lane(range.hi, e);
    const int row = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * ROWS;
    const int col = col_tile * COLS, rows = min(ROWS, hi - row), cols = min(COLS, p.N - col);
    const int64_t K = p.K, N = p.N;
    const float *a = static_cast<const float*>(p.rows) + row * K, *w = static_cast<const float*>(p.weight) + (e * N * K + (W_ACROSS ? col : col * K));
    float* out = static_cast<float*>(p.out) + row * N + col;
    const float* bias = !W_ACROSS && p.bias != nullptr ? static_cast<const float*>(p.bias) + e * N + col : nullptr;
    const int64_t ldw = W_ACROSS ? N : K;
    if constexpr (SMALL) small_tile<false, W_ACROSS>(a, K, rows, w, ldw, cols, p.K, out, N, nullptr, bias);
    else exact_tile(ExactOperand<false>{a, K, rows, p.K, {}}, ExactOperand<W_ACROSS>{w, ldw, cols, p.K, {}}, out, N, nullptr, bias);
}

// Parts of the reduction (blockIdx.y) go to [part][E_local][N,K] and sums to [part][E_local][N].
template <bool SMALL>
__global__ __launch_bounds__(256) void exact_weight_kernel(const WeightGradient p, int row_tiles, int col_tiles)
{
    const unsigned per_expert = static_cast<unsigned>(row_tiles) * static_cast<unsigned>(col_tiles);
    const int e = static_cast<int>(blockIdx.x / per_expert);
    const unsigned t = blockIdx.x % per_expert;
    constexpr int ROWS = SMALL ? small_rows(true) : kExactTile, COLS = SMALL ? kSmallCols : kExactTile;
    const int row = static_cast<int>(t / static_cast<unsigned>(col_tiles)) * ROWS, col = static_cast<int>(t % static_cast<unsigned>(col_tiles)) * COLS;
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int lo = wave_read_lane(range.lo, e), all = wave_read_lane(range.hi, e) - lo;
    const int stages = (all + kExactDepth - 1) / kExactDepth;
    const int first = static_cast<int>(static_cast<int64_t>(stages) * blockIdx.y / gridDim.y) * kExactDepth;
    const int n = max(min(all, static_cast<int>(static_cast<int64_t>(stages) * (blockIdx.y + 1) / gridDim.y) * kExactDepth) - first, 0);
    const int64_t N = p.N, K = p.K, begin = lo + first, at = static_cast<int64_t>(blockIdx.y) * p.E_local + e;
    const int rows = min(ROWS, p.N - row), cols = min(COLS, p.K - col);
    const float *a = static_cast<const float*>(p.dy) + begin * N + row, *w = static_cast<const float*>(p.x) + begin * K + col;
    float *out = static_cast<float*>(p.dw) + (at * N + row) * K + col, *sums = p.db != nullptr && col == 0 ? static_cast<float*>(p.db) + at * N + row : nullptr;
    if constexpr (SMALL) small_tile<true, true>(a, N, rows, w, K, cols, n, out, K, sums, nullptr);
    else exact_tile(ExactOperand<true>{a, N, rows, n, {}}, ExactOperand<true>{w, K, cols, n, {}}, out, K, sums, nullptr);
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


// Small tiles where larger ones would leave compute units without one.  Large and small, us, and how many large ones there are: gradients of rows 1024 rows, 8
// experts of 512 x 256 (96) 15.8 and 5.7; 2048, 8 of 1024 x 256 (160) 29.3 and 13.9; 8192, 8 of 512 x 128 (272) 16.4 and 14.2; 2048, 8 of 512 x 512 (320)
// 16.5 and 14.5; 4096 (576) 24.8 and 27.2.  Products, whose weights lie along the reduction, fall behind sooner: 512, 8 of 256 x 256 (64) 9.1 and 5.9; 1024, 8 of
// 512 x 256 (192) 9.3 and 8.7; but 2048, 8 of 512 x 512 (320) 16.5 and 22.6; 3000, 16 of 512 x 128 (496) 8.6 and 13.0; 4096, 8 of 512 x 512 (576) 24 and 42.
// Gradients of weights: 8192 rows, 8 of 512 x 128 (128) 18.7 and 18.1; 3000, 16 of 512 x 128 (256) 8.6 and 7.6; 2048, 8 of 512 x 512 (512) 15.1 and 21.3.
static bool small_tiles(int64_t large) { return large < 2 * 256; }

template <bool W_ACROSS>
static int launch_exact_rows(const ExactRows& p, hipStream_t stream, const char* fn)
{
    const int64_t most_experts = p.max_rows < p.E_local ? p.max_rows : p.E_local;
    auto tiles = [&](int64_t rows) { return (p.max_rows / rows + most_experts) * ((p.N + kExactTile - 1) / kExactTile); };
    const bool small = small_tiles(tiles(kExactTile));
    const int64_t grid = tiles(small ? small_rows(false) : kExactTile);
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "%s: too many tiles", fn);
    const int col_tiles = (p.N + kExactTile - 1) / kExactTile;
    if (small) hipLaunchKernelGGL((exact_rows_kernel<true, W_ACROSS>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p, col_tiles);
    else hipLaunchKernelGGL((exact_rows_kernel<false, W_ACROSS>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p, col_tiles);
    return EXF_OK;
}
int launch_exact_product(const ExactRows& p, hipStream_t stream) { return launch_exact_rows<false>(p, stream, "moe_grouped_product"); }
int launch_exact_rows_gradient(const ExactRows& p, hipStream_t stream) { return launch_exact_rows<true>(p, stream, "moe_grouped_product_dx"); }

// Parts of at least 256 rows until two workgroups a compute unit have one, at most 16.  us with parts of 128, 256 and 512 rows: 2048 rows, one expert of 256 x 256
// 13.9, 12.6, 12.8 (not split 20.0); 8192, 4 of 256 x 64 13.6, 12.3, 12.4; 2048, one of 64 x 64 12.5, 12.4, 14.3; but of few rows a second
// launch costs more than it saves: 512, one of 256 x 256 12.5, 12.6, 7.9; 2048, 4 of 256 x 64 12.5, 12.5, 7.9.  At most 8, 16 and 32 parts: 8192 rows, one of 64 x 64
// 16.0, 13.8, 17.5, 32768 rows 39.9, 26.0, 23.4 (not split 256).
static_assert(kSmallCols == kExactTile, "both kinds of tiles have as many columns");
static int64_t weight_tiles(int n, int k, int E_local, int rows) { return static_cast<int64_t>(E_local) * ((n + rows - 1) / rows) * ((k + kExactTile - 1) / kExactTile); }
int exact_weight_gradient_splits(int64_t A, int n, int k, int E_local)
{
    const bool small = small_tiles(weight_tiles(n, k, E_local, kExactTile));
    const int64_t wanted = 512 / weight_tiles(n, k, E_local, small ? small_rows(true) : kExactTile), most = A / (256 * E_local);
    const int64_t s = wanted < most ? wanted : most;
    return static_cast<int>(s < 2 ? 1 : (s > 16 ? 16 : s));
}
int launch_exact_weight_gradient(const WeightGradient& g, hipStream_t stream)
{
    const bool small = small_tiles(weight_tiles(g.N, g.K, g.E_local, kExactTile));
    const int tile_rows = small ? small_rows(true) : kExactTile;
    const int64_t grid = weight_tiles(g.N, g.K, g.E_local, tile_rows), each = static_cast<int64_t>(g.E_local) * g.N * g.K;
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_dw: too many tiles");
    const int splits = exact_weight_gradient_splits(g.max_rows, g.N, g.K, g.E_local);
    float* parts = static_cast<float*>(g.workspace);
    WeightGradient p = g;
    if (splits > 1) {
        p.dw = parts;
        if (p.db != nullptr) p.db = parts + splits * each;
    }
    const dim3 blocks(static_cast<unsigned>(grid), static_cast<unsigned>(splits));
    const int rows = (g.N + tile_rows - 1) / tile_rows, cols = (g.K + kExactTile - 1) / kExactTile;
    if (small) hipLaunchKernelGGL(exact_weight_kernel<true>, blocks, dim3(256), 0, stream, p, rows, cols);
    else hipLaunchKernelGGL(exact_weight_kernel<false>, blocks, dim3(256), 0, stream, p, rows, cols);
    if (splits == 1) return EXF_OK;
    return launch_join_parts(parts, each, g.dw, parts + splits * each, g.db != nullptr ? static_cast<int64_t>(g.E_local) * g.N : 0, g.db, splits, EXF_F32, stream);
}

}  // namespace exf
