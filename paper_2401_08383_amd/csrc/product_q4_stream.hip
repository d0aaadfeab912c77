// moe_grouped_product_q4, bf16, weights that fill the chip: operands staged through LDS.
//
// A lane of the matrix instruction needs 16 bytes of its own column, and neighbouring lanes have different columns: loaded straight to registers every lane is
// an access of its own to the L1, 64 a load, and the L1 is the bound.  Copied to LDS first, in units of 256 elements - 128 bytes of a column, 512 of a row -
// neighbouring lanes fetch what lies together, and a load of a wavefront is 16 accesses.  Pieces of 16 bytes trade places inside a column's (row's) part of a
// unit so that the 16 lanes that read one piece each of 16 columns (rows) meet all banks once.
//   A workgroup has 16 R rows and 4 x 16 C columns of an expert, a wavefront all rows and 16 C of the columns, with two slots of codes, scales and zero points of
// its own; the rows' two are shared by four wavefronts, each copies a quarter of the rows there are (what a slot holds of others goes into sums that are not
// stored).  One barrier a unit: behind it the unit is there for all, and the slot of the unit before is free.  Where columns are too few to fill the chip, KS times
// four wavefronts take every KS-th unit each, and their sums are added in order.
//   ODD: K ends inside a unit.  Its groups past the end are left out; a column's scales and zero points begin anywhere in a word of four bytes.
#include "q4.hpp"

namespace exf {

template <int GROUP, int U, int R, int C, int KS, bool ODD, bool ZERO>
struct Q4Ring {
    static constexpr int kUnit = U, kSteps = U / 128, kGroups = kUnit / GROUP, kColumns = 16 * C;
    // words of a column's unit, that hold its scales and its zero points; ODD: they begin anywhere in the first
    static constexpr int kScaleWords = ODD ? kGroups / 2 + 1 : (kGroups + 1) / 2, kZeroWords = ODD ? (kGroups + 2) / 4 + 1 : (kGroups + 3) / 4;
    static constexpr bool kWide = !ODD && kScaleWords == 4;  // 16 bytes at once
    static constexpr int kCodes = kColumns * kUnit / 2, kScales = kColumns * kScaleWords * 4, kZeros = ZERO ? kColumns * kZeroWords * 4 : 0, kRows = 16 * R * kUnit * 2;
    static constexpr int kWave64 = kCodes + kScales + kZeros;  // bytes of a unit of a wavefront
    static constexpr int kCodeLoads = kCodes / 1024, kRowLoads = kRows / 4096;
    static constexpr int kScaleLanes = kWide ? kColumns : kColumns * kScaleWords, kScaleLoads = (kScaleLanes + 63) / 64;
    static constexpr int kZeroLanes = kColumns * kZeroWords, kZeroLoads = ZERO ? (kZeroLanes + 63) / 64 : 0;
    static constexpr int kBytes = KS * 2 * (kRows + 4 * kWave64);
};

// Words from byte `at` (0 to 3) of the first on.
template <int N>
__device__ __forceinline__ void from_byte(uint32_t (&w)[N], uint32_t at)
{
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = __builtin_amdgcn_alignbyte(i + 1 < N ? w[i + 1] : 0u, w[i], at);
}

template <int GROUP, int U, int R, int C, int KS, bool PAST, bool ODD, bool ZERO>
__global__ __launch_bounds__(256 * KS, KS > 2 ? KS : 2) void q4_stream_kernel(const Q4Product p, int col_tiles)
{
    using Ring = Q4Ring<GROUP, U, R, C, KS, ODD, ZERO>;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const uint32_t smem_addr = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));
    const int lane = lane_id(), in16 = lane & 15, quad = lane >> 4, nth = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wave = nth % 4, share = nth / 4;
    const ExpertRows range = expert_rows(p.offsets, p.E_local, p.max_rows);
    const int tiles = (range.hi - range.lo + 16 * R - 1) / (16 * R), upto = wave_inclusive_scan(tiles);
    const int64_t N = p.N;
    const int groups = p.K / GROUP;
    const int units = (p.K + Ring::kUnit - 1) / Ring::kUnit, turns = (units + KS - 1) / KS, own = (units - share + KS - 1) / KS;
    const uint32_t rows_at = smem_addr + share * (2 * Ring::kRows), mine_at = smem_addr + KS * 2 * Ring::kRows + nth * (2 * Ring::kWave64);
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
        // (Products of 24 bits: the wider form writes a scalar register pair too, which the loads that follow, in assembly, must not read at once.)
        static_assert(EXF_MAX_PRODUCT_WIDTH <= 1 << 22, "twice a reduction has 24 bits");
        uint32_t code_at[Ring::kCodeLoads], row_at[Ring::kRowLoads];
#pragma unroll
        for (int i = 0; i < Ring::kCodeLoads; ++i) {
            constexpr int kPieces = U / 32;  // of a column
            const int c = i * (64 / kPieces) + lane / kPieces;
            code_at[i] = __umul24(max(min(c, cols - 1), 0), p.K / 2) + ((lane ^ (c / (16 / kPieces))) % kPieces) * 16;
        }
#pragma unroll
        for (int i = 0; i < Ring::kRowLoads; ++i) {
            constexpr int kPieces = U / 8;  // of a row
            const int r = (i * 4 + wave) * (64 / kPieces) + lane / kPieces;
            row_at[i] = __umul24(min(r, rows - 1), p.K * 2) + ((lane % kPieces) ^ (r & 15)) * 16;
        }
        // What a unit has behind the end of a column or row is the next one's, and not used; of the last ones of all it is the last piece there is.
        const int64_t cols_left = p.E_local * N - first_col, rows_left = p.max_rows - lo;
        auto within = [&](uint32_t at, int64_t bytes) { return ODD ? min(at, static_cast<uint32_t>(bytes < 0x7fffffff ? bytes : 0x7fffffff)) : at; };
        auto issue = [&](int t) {
            const int u = t * KS + share, slot = t % 2;
            const uint32_t mine = mine_at + slot * Ring::kWave64;
#pragma unroll
            for (int i = 0; i < Ring::kCodeLoads; ++i) {
                const uint32_t at = within(code_at[i], cols_left * (p.K / 2) - u * (Ring::kUnit / 2) - 16);
                if constexpr (PAST) lds_dma_16B_stream(codes + u * (Ring::kUnit / 2), at, mine + i * 1024);
                else lds_dma_16B(codes + u * (Ring::kUnit / 2), at, mine + i * 1024);
            }
#pragma unroll
            for (int i = 0; i < Ring::kRowLoads; ++i)
                if ((i * 4 + wave) * (512 / U) < rows)
                    lds_dma_16B(x + u * (Ring::kUnit * 2), within(row_at[i], rows_left * (p.K * 2) - u * (Ring::kUnit * 2) - 16), rows_at + slot * Ring::kRows + (i * 4 + wave) * 1024);
#pragma unroll
            for (int i = 0; i < Ring::kScaleLoads; ++i) {
                const int l = i * 64 + lane;
                if (l < Ring::kScaleLanes) {
                    const uint32_t column = __umul24(max(min(Ring::kWide ? l : l / Ring::kScaleWords, cols - 1), 0), groups * 2);
                    if constexpr (Ring::kWide) lds_dma_16B(scales + u * 16, column, mine + Ring::kCodes + i * 1024);
                    else lds_dma_4B(scales, within((column + u * Ring::kGroups * 2 + l % Ring::kScaleWords * 4) & ~3u, cols_left * groups * 2 - 4), mine + Ring::kCodes + i * 256);
                }
            }
            if constexpr (ZERO)
#pragma unroll
                for (int i = 0; i < Ring::kZeroLoads; ++i) {
                    const int l = i * 64 + lane;
                    if (l < Ring::kZeroLanes) {
                        const uint32_t at = __umul24(max(min(l / Ring::kZeroWords, cols - 1), 0), groups) + u * Ring::kGroups + l % Ring::kZeroWords * 4;
                        lds_dma_4B(zeros, within(at & ~3u, cols_left * groups - 4), mine + Ring::kCodes + Ring::kScales + i * 256);
                    }
                }
        };
        // What this wavefront copied of the rows, in the order of the codes, once for the four that share it: 421 us for 428 (512 rows over 64 of 16384 x 4096), 387 for 397
        // (64 rows).  Otherwise each puts what it multiplies in order: where it has 64 columns (512 rows over 8 of 4096 x 4096 in such tiles 39.5, once 44) or shares the reduction
        // (7 over 3 of 13232 x 15488 97, once 120), and where there are 32 rows (512 over 8 of 4096 x 4096 39.8, once 41.7).
        constexpr bool kOnce = R == 1 && KS == 1;
        auto put_in_order = [&](int t) {
#pragma unroll
            for (int i = 0; i < Ring::kRowLoads; ++i)
                if ((i * 4 + wave) * (512 / U) < rows) {
                    unsigned char* const at = smem + (share * 2 + t % 2) * Ring::kRows + (i * 4 + wave) * 1024 + lane * 16;
                    const bf16x8_t v = in_code_order(*reinterpret_cast<const uint4*>(at));
                    __builtin_memcpy(__builtin_assume_aligned(at, 16), &v, 16);
                }
        };
        f32x4_t total[R][C];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) total[r][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        auto multiply = [&](int t) {
            const int u = t * KS + share, slot = t % 2;
            const unsigned char *mine = smem + KS * 2 * Ring::kRows + nth * (2 * Ring::kWave64) + slot * Ring::kWave64, *shared = smem + (share * 2 + slot) * Ring::kRows;
            float scale[C][Ring::kGroups], zero[C][Ring::kGroups];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint32_t first = __umul24(max(min(c * 16 + in16, cols - 1), 0), groups) + u * Ring::kGroups;
                uint32_t s[Ring::kScaleWords], z[Ring::kZeroWords];
                __builtin_memcpy(s, __builtin_assume_aligned(mine + Ring::kCodes + (c * 16 + in16) * Ring::kScaleWords * 4, ODD ? 4 : Ring::kScaleWords * 4), sizeof(s));
                if constexpr (ODD || Ring::kGroups == 1) from_byte(s, (first & 1u) * 2);
                if constexpr (ZERO) {
                    __builtin_memcpy(z, __builtin_assume_aligned(mine + Ring::kCodes + Ring::kScales + (c * 16 + in16) * Ring::kZeroWords * 4, ODD ? 4 : Ring::kZeroWords * 4), sizeof(z));
                    if constexpr (ODD || Ring::kGroups < 4) from_byte(z, first & 3u);
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
                    if (ODD && u * Ring::kGroups + h * (128 / GROUP) + g >= groups) continue;  // (the end of the columns)
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
                            const uint4 v = *reinterpret_cast<const uint4*>(shared + (r * 16 + in16) * (U * 2) + (h * 16 + (piece ^ in16)) * 16);
                            a[r] = kOnce ? as_bf16x8(v.x, v.y, v.z, v.w) : in_code_order(v);
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
        if (KS == 1 || own > 0) issue(0);
        for (int t = 0; t < turns; ++t) {
            wait_vmcnt<0>();
            if (kOnce) put_in_order(t);
            barrier_for_lds();
            if (t + 1 < own) issue(t + 1);
            if (KS == 1 || t < own) multiply(t);
        }
        if constexpr (KS > 1) {  // the shares' sums, in their order
            static_assert(R == 1, "a tile of rows");
            f32x4_t* const parts = reinterpret_cast<f32x4_t*>(smem) + wave * ((KS - 1) * C * kWave) + lane;
            barrier_for_lds();
            if (share > 0)
#pragma unroll
                for (int c = 0; c < C; ++c) parts[((share - 1) * C + c) * kWave] = total[0][c];
            barrier_for_lds();
            if (share == 0)
#pragma unroll
                for (int s = 1; s < KS; ++s)
#pragma unroll
                    for (int c = 0; c < C; ++c) total[0][c] += parts[((s - 1) * C + c) * kWave];
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = c * 16 + in16;
            if (at >= cols || (KS > 1 && share > 0)) continue;
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

// What the choice goes by: tiles, were the rows spread evenly over the experts that can have any.  The host knows how many rows there are, not whose, nor how many lie outside all
// ranges.  us, even, nine tenths of them one expert's, and all of one expert in eight: 512, 64, 16384 x 4096 415, 499 and 215; 1280, 64, 4096 x 4096 155, 216 and 92; 2048, 32, 4096 x 2048 58, 90
// and 50; 8192, 8, 4096 x 4096 355, 381 and 349.  Seven eighths of the rows outside, and a call with the others alone: 512, 64 396 and 392; 1280, 64 152 and 115; 2048, 32 65 and 46.
struct Q4Spread {
    int64_t experts, mean;
    int N;
    Q4Spread(int64_t A, int n, int E_local) : experts(A < E_local ? A : E_local), mean((A + experts - 1) / experts), N(n) {}
    int64_t of_rows(int rows) const { return (mean + rows - 1) / rows; }  // of an expert
    int64_t workgroups(int rows, int cols) const { return experts * of_rows(rows) * ((N + cols - 1) / cols); }
};

// (Times of single calls are in a graph or back to back, which differ by less than boxes and moments do: 512, 64, 16384 x 4096 411 to 431.)
// Workgroups for two thirds of the compute units; half of that where a tile has more than 8 rows, which the other kernel loads over and over.  Streamed and not, us (rows,
// experts, columns x reduction): 512, 64, 16384 x 4096 411 and 946; 1024, 64, 4096 x 1056 57 and 96; 1, 1, 16384 x 4096 11.4 and 15.3; 43, 10, 1200 x 4096 10.9 and 13.5;
// 100, 6, 512 x 8192 16.4 and 23.2; but 8, 8, 1024 x 4096 10.5 and 9.1; 16, 1, 4096 x 4096 10.2 and 8.5; 1, 1, 4096 x 1024 5.3 and 4.5; 66, 4, 352 x 10624 22 and 15.8.
bool q4_streams(int64_t A, int n, int E_local)
{
    const Q4Spread s(A, n, E_local);
    return s.workgroups(16, 64) * (s.mean > 8 ? 2 : 1) >= 160;
}

// Tiles, rows x columns, us, as above.
//   64 x 256, units of 128, where the rows fill them and two workgroups a compute unit are left (what turns codes into numbers is shared by the rows), not 32 x 256: 8192, 8, 4096 x 4096
// 353 and 419; 2048, 32, 4096 x 2048 70 and 76; but 1500, 1, 4096 x 4096 94 and 92 (82 to 92 since); 2048, 40, 4096 x 2048 (51 rows of 64) 98 and 93.
//   32 x 256, units of 128 so that three fit a compute unit, for nearly that many, not 32 x 128: 1500, 1, 4096 x 4096 86 and 98; 1500, 16, 4096 x 2048 48 and 55; but 600, 2, 8192 x 8192
// 207 and 183; 1280, 64, 4096 x 4096 213 and 153.
//   32 x 128 where an expert has more than 16 rows, not 16 x 128: 1280, 64, 16384 x 4096 608 and 717; 512, 16, 4096 x 4096 37 and 47; 256, 8, 4096 x 4096 24.6 and 27.1; but from 160
// workgroups on, with fewer 16 x 64: 80, 3, 8192 x 4096 24.5 and 25.2; 200, 8, 2048 x 2048 17.5 and 13.0.
//   16 x 64 with two shares of the reduction while 16 x 128 has less than one and a half workgroups a compute unit: 5, 5, 8192 x 4096 22.9 and 23.8; 10, 10, 4096 x 4096 28.9 and 34.3; but 12, 12,
// 4096 x 2048 14.7 and 14.2; 115, 2, 7488 x 128 9.1 and 6.2.  With four shares while they are one a compute unit and a share has some units: 1, 1, 16384 x 16384 29.6 and 34.3;
// 43, 10, 1200 x 4096 10.9 and 11.7; but 4, 4, 4096 x 1024 6.0 and 5.5.
//   A third slot in LDS gained nothing (12.2 for 12.2, 17.7 for 17.1, 488 for 433).
//   Weights that are read once and that the 256 MB behind the L2 cannot hold until the next call go past the caches: 411 us for 512, 64, 16384 x 4096, 426 otherwise (64 rows: 385 and 402; 1280
// rows 588 and 608); weights that it can hold do not, 31.2 and 36.1 (1024, 64, 4096 x 1024, called again and again).
int launch_q4_stream(const Q4Product& p, int group, hipStream_t stream)
{
    int rc = EXF_OK;
    auto run = [&](auto size, auto unit, auto row_tiles, auto col_tiles, auto shares, auto past, auto odd, auto zero) {
        constexpr int G = decltype(size)::value, U = decltype(unit)::value, R = decltype(row_tiles)::value, C = decltype(col_tiles)::value, KS = decltype(shares)::value;
        constexpr bool PAST = decltype(past)::value, ODD = decltype(odd)::value, ZERO = decltype(zero)::value;
        constexpr size_t lds = Q4Ring<G, U, R, C, KS, ODD, ZERO>::kBytes;
        static_assert(lds <= 160 * 1024, "a CU has 160 KiB");
        const int64_t cols = (p.N + 64 * C - 1) / (64 * C), grid = (p.max_rows / (16 * R) + (p.max_rows < p.E_local ? p.max_rows : p.E_local)) * cols;
        auto kern = q4_stream_kernel<G, U, R, C, KS, PAST, ODD, ZERO>;
        static std::atomic<uint64_t> allowed{0};
        rc = allow_lds(reinterpret_cast<const void*>(kern), lds, allowed, "moe_grouped_product_q4");
        if (rc == EXF_OK) hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid < (1 << 22) ? grid : 1 << 22)), dim3(256 * KS), lds, stream, p, static_cast<int>(cols));
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 128> step;
    const std::integral_constant<int, 256> steps;
    const std::true_type yes;
    const std::false_type no;
    const Q4Spread s(p.max_rows, p.N, p.E_local);
    const bool tallest = s.mean > 48 && s.workgroups(64, 256) >= 512 && 8 * s.mean >= 7 * 64 * s.of_rows(64), tall = s.mean > 48 && s.workgroups(32, 256) >= 700;
    const bool two_tiles = s.mean > 16 && s.workgroups(32, 128) >= 160, few = s.workgroups(16, 64) <= 768, fewest = s.workgroups(16, 64) <= 256 && p.K >= 2048;
    const bool past = s.mean <= 32 && static_cast<int64_t>(p.E_local) * p.N * p.K / 2 > (int64_t{256} << 20);
    pick_q4_group(group, [&](auto size) {
        auto with = [&](auto zero) {
            auto ends = [&](auto unit, auto run_with) {
                if constexpr (decltype(unit)::value > decltype(size)::value)
                    if (p.K % decltype(unit)::value != 0) return run_with(yes);
                run_with(no);  // (a unit that is a group always fits)
            };
            if (tallest) ends(step, [&](auto odd) { run(size, step, four, four, one, no, odd, zero); });
            else if (tall) ends(step, [&](auto odd) { run(size, step, two, four, one, no, odd, zero); });
            else if (two_tiles && past) ends(steps, [&](auto odd) { run(size, steps, two, two, one, yes, odd, zero); });
            else if (two_tiles) ends(steps, [&](auto odd) { run(size, steps, two, two, one, no, odd, zero); });
            else if (fewest) ends(steps, [&](auto odd) { run(size, steps, one, one, four, no, odd, zero); });
            else if (few) ends(steps, [&](auto odd) { run(size, steps, one, one, two, no, odd, zero); });
            else if (past) ends(steps, [&](auto odd) { run(size, steps, one, two, one, yes, odd, zero); });
            else ends(steps, [&](auto odd) { run(size, steps, one, two, one, no, odd, zero); });
        };
        if (p.zero != nullptr) with(yes);
        else with(no);
    });
    return rc;
}

}  // namespace exf
