// moe_grouped_product_q4, bf16, weights that fill the chip: operands staged through LDS.
//
// A lane of the matrix instruction needs 16 bytes of its own column, and neighbouring lanes have different columns: loaded straight to registers every lane is
// an access of its own to the L1, 64 a load, and the L1 is the bound.  Copied to LDS first, in units of 256 elements - 128 bytes of a column, 512 of a row -
// neighbouring lanes fetch what lies together, and a load of a wavefront is 16 accesses.  Pieces of 16 bytes trade places inside a column's (row's) part of a
// unit so that the 16 lanes that read one piece each of 16 columns (rows) meet all banks once.
//   A workgroup has 16 R rows and 4 x 16 C columns of an expert, a wavefront all rows and 16 C of the columns, with two slots of codes, scales and
// zero points of its own; the rows' two are shared, each wavefront copies a quarter of the rows there are (what a slot holds of others goes into sums that are not
// stored).  One barrier a unit: behind it the unit is there for all, and the slot of the unit before is free.
#include "q4.hpp"

namespace exf {

template <int GROUP, int U, int R, int C, bool ZERO>
struct Q4Ring {
    static constexpr int kUnit = U, kSteps = U / 128, kGroups = kUnit / GROUP, kColumns = 16 * C;
    // words of a column's unit, that hold its scales and its zero points
    static constexpr int kScaleWords = (kGroups + 1) / 2, kZeroWords = (kGroups + 3) / 4;
    static constexpr int kCodes = kColumns * kUnit / 2, kScales = kColumns * kScaleWords * 4, kZeros = ZERO ? kColumns * kZeroWords * 4 : 0, kRows = 16 * R * kUnit * 2;
    static constexpr int kWave64 = kCodes + kScales + kZeros;  // bytes of a unit of a wavefront
    static constexpr int kCodeLoads = kCodes / 1024, kRowLoads = kRows / 4096;
    static constexpr int kScaleLanes = kScaleWords == 4 ? kColumns : kColumns * kScaleWords, kScaleLoads = (kScaleLanes + 63) / 64;
    static constexpr int kZeroLanes = kColumns * kZeroWords, kZeroLoads = ZERO ? (kZeroLanes + 63) / 64 : 0;
    static constexpr int kBytes = 2 * (kRows + 4 * kWave64);
};

template <int GROUP, int U, int R, int C, bool PAST, bool ZERO>
__global__ __launch_bounds__(256, 2) void q4_stream_kernel(const Q4Product p, int col_tiles)
{
    using Ring = Q4Ring<GROUP, U, R, C, ZERO>;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const uint32_t smem_addr = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));
    const int lane = lane_id(), in16 = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + 16 * R - 1) / (16 * R), upto = wave_inclusive_scan(tiles);
    const int64_t N = p.N, groups = p.K / GROUP;
    const int units = p.K / Ring::kUnit;
    const uint32_t rows_at = smem_addr, mine_at = smem_addr + 2 * Ring::kRows + wave * (2 * Ring::kWave64);
    const CodeBits bits = code_bits();
    for (int64_t tile = blockIdx.x;; tile += gridDim.x) {
        const int row_tile = static_cast<int>(tile / col_tiles);
        const unsigned long long owner = __ballot(row_tile < upto);
        if (owner == 0ull) return;  // (the same for all wavefronts)
        const int e = __builtin_ctzll(owner), lo = wave_read_lane(range.lo, e) + (row_tile - wave_read_lane(upto - tiles, e)) * 16 * R;
        const int rows = min(16 * R, wave_read_lane(range.hi, e) - lo);
        const int col0 = (static_cast<int>(tile % col_tiles) * 4 + wave) * Ring::kColumns, cols = min(Ring::kColumns, p.N - col0);  // (none: column 0 is loaded)
        const int64_t first_col = e * N + (col0 < p.N ? col0 : 0);
        const unsigned char* codes = uniform_ptr(p.weight + first_col * (p.K / 2));
        const unsigned char* scales = uniform_ptr(static_cast<const unsigned char*>(p.scale) + first_col * groups * 2);
        const unsigned char* zeros = uniform_ptr(ZERO ? p.zero + first_col * groups : nullptr);
        const unsigned char* x = uniform_ptr(static_cast<const unsigned char*>(p.rows) + static_cast<int64_t>(lo) * p.K * 2);
        uint32_t code_at[Ring::kCodeLoads], row_at[Ring::kRowLoads];
#pragma unroll
        for (int i = 0; i < Ring::kCodeLoads; ++i) {
            constexpr int kPieces = U / 32;  // of a column
            const int c = i * (64 / kPieces) + lane / kPieces;
            code_at[i] = static_cast<uint32_t>(max(min(c, cols - 1), 0)) * static_cast<uint32_t>(p.K / 2) + ((lane ^ (c / (16 / kPieces))) % kPieces) * 16;
        }
#pragma unroll
        for (int i = 0; i < Ring::kRowLoads; ++i) {
            constexpr int kPieces = U / 8;  // of a row
            const int r = (i * 4 + wave) * (64 / kPieces) + lane / kPieces;
            row_at[i] = static_cast<uint32_t>(min(r, rows - 1)) * static_cast<uint32_t>(p.K * 2) + ((lane % kPieces) ^ (r & 15)) * 16;
        }
        auto issue = [&](int u) {
            const int slot = u % 2;
            const uint32_t mine = mine_at + slot * Ring::kWave64;
#pragma unroll
            for (int i = 0; i < Ring::kCodeLoads; ++i) {
                if constexpr (PAST) lds_dma_16B_stream(codes + u * (Ring::kUnit / 2), code_at[i], mine + i * 1024);
                else lds_dma_16B(codes + u * (Ring::kUnit / 2), code_at[i], mine + i * 1024);
            }
#pragma unroll
            for (int i = 0; i < Ring::kRowLoads; ++i)
                if ((i * 4 + wave) * (512 / U) < rows) lds_dma_16B(x + u * (Ring::kUnit * 2), row_at[i], rows_at + slot * Ring::kRows + (i * 4 + wave) * 1024);
#pragma unroll
            for (int i = 0; i < Ring::kScaleLoads; ++i) {
                const int l = i * 64 + lane;
                if (l < Ring::kScaleLanes) {
                    const uint32_t mine_of = static_cast<uint32_t>(max(min(Ring::kScaleWords == 4 ? l : l / Ring::kScaleWords, cols - 1), 0)) * static_cast<uint32_t>(groups * 2);
                    if constexpr (Ring::kScaleWords == 4) lds_dma_16B(scales + u * 16, mine_of, mine + Ring::kCodes + i * 1024);
                    else lds_dma_4B(scales, (mine_of + u * Ring::kGroups * 2 + l % Ring::kScaleWords * 4) & ~3u, mine + Ring::kCodes + i * 256);
                }
            }
            if constexpr (ZERO)
#pragma unroll
                for (int i = 0; i < Ring::kZeroLoads; ++i) {
                    const int l = i * 64 + lane;
                    if (l < Ring::kZeroLanes) {
                        const uint32_t at = static_cast<uint32_t>(max(min(l / Ring::kZeroWords, cols - 1), 0)) * static_cast<uint32_t>(groups) + u * Ring::kGroups + l % Ring::kZeroWords * 4;
                        lds_dma_4B(zeros, at & ~3u, mine + Ring::kCodes + Ring::kScales + i * 256);
                    }
                }
        };
        f32x4_t total[R][C];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) total[r][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        auto multiply = [&](int u) {
            const int slot = u % 2;
            const unsigned char *mine = smem + 2 * Ring::kRows + wave * (2 * Ring::kWave64) + slot * Ring::kWave64, *shared = smem + slot * Ring::kRows;
            float scale[C][Ring::kGroups], zero[C][Ring::kGroups];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint32_t first = static_cast<uint32_t>(max(min(c * 16 + in16, cols - 1), 0)) * static_cast<uint32_t>(groups) + u * Ring::kGroups;
                uint32_t s[Ring::kScaleWords], z[Ring::kZeroWords];
                __builtin_memcpy(s, __builtin_assume_aligned(mine + Ring::kCodes + (c * 16 + in16) * Ring::kScaleWords * 4, Ring::kScaleWords * 4), sizeof(s));
                if constexpr (Ring::kGroups == 1) s[0] >>= (first & 1u) * 16;  // (the one of the word's two)
                if constexpr (ZERO) {
                    __builtin_memcpy(z, __builtin_assume_aligned(mine + Ring::kCodes + Ring::kScales + (c * 16 + in16) * Ring::kZeroWords * 4, Ring::kZeroWords * 4), sizeof(z));
                    if constexpr (Ring::kGroups < 4) z[0] >>= (first & 3u) * 8;  // (those of the word's four)
                }
#pragma unroll
                for (int g = 0; g < Ring::kGroups; ++g) {
                    scale[c][g] = __uint_as_float(g % 2 == 0 ? s[g / 2] << 16 : s[g / 2] & 0xffff0000u);
                    zero[c][g] = ZERO ? static_cast<float>((z[g / 4] >> (g % 4 * 8)) & 255u) : 8.0f;
                }
            }
            constexpr bool TURN = GROUP < 128;
#pragma unroll
            for (int h = 0; h < Ring::kSteps; ++h) {
                uint32_t w[C][4];
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const uint4 v = *reinterpret_cast<const uint4*>(mine + (c * 16 + in16) * (U / 2) + (((h * 4 + quad) ^ (in16 / (512 / U))) % (U / 32)) * 16);
                    w[c][0] = v.x, w[c][1] = v.y, w[c][2] = v.z, w[c][3] = v.w;
                    if constexpr (TURN) turn_quads(w[c]);
                }
#pragma unroll
                for (int g = 0; g < 128 / GROUP; ++g) {
                    f32x4_t sum[R][C], sum_x[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        sum_x[r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int c = 0; c < C; ++c) sum[r][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    }
#pragma unroll
                    for (int m = g * (GROUP / 32); m < (g + 1) * (GROUP / 32); ++m) {
                        bf16x8_t a[R];
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const int piece = TURN ? m * 4 + quad : quad * 4 + m;
                            a[r] = in_code_order(*reinterpret_cast<const uint4*>(shared + (r * 16 + in16) * (U * 2) + (h * 16 + (piece ^ in16)) * 16));
                            sum_x[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[r], ones_bf16(), sum_x[r], 0, 0, 0);
                        }
#pragma unroll
                        for (int c = 0; c < C; ++c) {
                            const bf16x8_t b = codes_bf16(w[c][m], bits);
#pragma unroll
                            for (int r = 0; r < R; ++r) sum[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[r], b, sum[r][c], 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const float s = scale[c][h * (128 / GROUP) + g], less = -(16.0f + zero[c][h * (128 / GROUP) + g]);
#pragma unroll
                        for (int r = 0; r < R; ++r)
#pragma unroll
                            for (int q = 0; q < 4; ++q) total[r][c][q] = fmaf(s, fmaf(less, sum_x[r][q], sum[r][c][q]), total[r][c][q]);
                    }
                }
            }
        };
        issue(0);
        for (int u = 0; u < units; ++u) {
            wait_vmcnt<0>();
            barrier_for_lds();
            if (u + 1 < units) issue(u + 1);
            multiply(u);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = c * 16 + in16;
            if (at >= cols) continue;
            const float b = p.bias != nullptr ? bf16_to_f32(static_cast<const bf16_t*>(p.bias)[first_col + at]) : 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = r * 16 + quad * 4 + q;
                    if (row < rows) static_cast<bf16_t*>(p.out)[(lo + row) * N + col0 + at] = f32_to_bf16(total[r][c][q] + b);
                }
        }
        barrier_for_lds();
    }
}

// Whole steps of 128 elements, and workgroups of 128 columns for half of the compute units at least.  Streamed and not, us: 512 rows over 64 experts of 16384 x
// 4096 411 and 946, 64 rows 385 and 715; one row, 16384 x 4096 13.2 and 14; 8 over 8 of 4096 x 1024 6.4 and 9.5; one of 4096 x 1024 4.9 and 3.9; 16 over 2 of 2048 x
// 8192 22 and 12.5.
bool q4_streams(int64_t A, int n, int k, int E_local) { return k % 128 == 0 && (n + 127) / 128 * (A < E_local ? A : E_local) >= 128; }

// Tiles, us.  Few rows a tile read the weights once (1024 rows over 64 experts of 4096 x 1024: 31.6 with 16 x 128 a workgroup, 39.1 with 32 x 256), many share
// what it costs to turn codes into numbers (2048 rows over the same 49.6 and 43.7; over 8 of 4096 x 4096 157.7 and 114.7).  Units of 256 elements are a whole line
// of a column; those of 128 are for the columns that end inside one (512 rows over 64 of 16384 x 4096: 433 and 557).  A third slot in LDS costs a workgroup a
// compute unit (488).  Weights that the 256 MB behind the L2 cannot hold until the next call go past the caches: 411 us for 512 rows over 64 of 16384 x 4096, 426
// otherwise (64 rows: 385 and 402); weights that it can hold do not, 31.2 and 36.1 (1024 rows over 64 of 4096 x 1024, called again and again).
int launch_q4_stream(const Q4Product& p, int group, hipStream_t stream)
{
    int rc = EXF_OK;
    auto run = [&](auto size, auto unit, auto row_tiles, auto col_tiles, auto past, auto zero) {
        constexpr int G = decltype(size)::value, U = decltype(unit)::value, R = decltype(row_tiles)::value, C = decltype(col_tiles)::value;
        constexpr bool PAST = decltype(past)::value, ZERO = decltype(zero)::value;
        constexpr size_t lds = Q4Ring<G, U, R, C, ZERO>::kBytes;
        static_assert(lds <= 160 * 1024, "a CU has 160 KiB");
        const int64_t cols = (p.N + 64 * C - 1) / (64 * C), grid = (p.max_rows / (16 * R) + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
        auto kern = q4_stream_kernel<G, U, R, C, PAST, ZERO>;
        static std::atomic<uint64_t> allowed{0};
        rc = allow_lds(reinterpret_cast<const void*>(kern), lds, allowed, "moe_grouped_product_q4");
        if (rc == EXF_OK) hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid < (1 << 22) ? grid : 1 << 22)), dim3(256), lds, stream, p, static_cast<int>(cols));
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 128> step;
    const std::integral_constant<int, 256> steps;
    const int64_t mean = p.max_rows / p.E_local, bytes = static_cast<int64_t>(p.E_local) * p.N * p.K / 2;
    pick_q4_group(group, [&](auto size) {
        auto with = [&](auto zero) {
            if (mean > 24) run(size, step, two, four, std::false_type(), zero);
            else if (p.K % 256 != 0) run(size, step, one, two, std::false_type(), zero);
            else if (bytes > (int64_t{256} << 20)) run(size, steps, one, two, std::true_type(), zero);
            else run(size, steps, one, two, std::false_type(), zero);
        };
        if (p.zero != nullptr) with(std::true_type());
        else with(std::false_type());
    });
    return rc;
}

}  // namespace exf
