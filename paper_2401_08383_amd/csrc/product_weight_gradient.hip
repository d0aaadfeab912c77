// Weight gradient of the experts' products in tiles, bf16 (see product_tiles.hpp): dw[e][N,K] = dy[rows of e, N]^T x[rows of e, K].
//
// The reduction is an expert's rows, so all tiles of an expert take equally long; the longest experts come first.  An XCD takes 32
// consecutive tiles at a time, one for each compute unit: four rows of tiles by eight columns, which share their operands in its L2.
//   Long reductions: a workgroup a tile.  Few tiles: the reduction is split, the parts' sums go to the workspace in fp32, and a
//   second launch adds them up in order.
//   Short ones, a stage or a few with as many outputs as weights: a workgroup is there for good and its tiles are one stream
//   of stages; while a tile is multiplied and its results stored, the stages of the next ones are on their way.
#include "product_tiles.hpp"

namespace exf {

constexpr int kGroupTiles = 32, kGroupRows = 4;

struct WeightTiles {
    const bf16_t *dy, *x;
    const int32_t* offsets;
    void* out;          // [splits][E_local][N,K]
    void* sums;         // [splits][E_local][N] or null: of dy over the rows (tiles of the first columns multiply by ones as well)
    int max_rows, N, K, E_local, splits;
};

// Quotient of wavefront-uniform numbers below 2^24 through the divisor's reciprocal, with a correction.
__device__ __forceinline__ unsigned quotient(unsigned n, unsigned d, float reciprocal)
{
    int q = static_cast<int>(static_cast<float>(n) * reciprocal);
    const int r = static_cast<int>(n) - q * static_cast<int>(d);
    q += r < 0 ? -1 : (r >= static_cast<int>(d) ? 1 : 0);
    return static_cast<unsigned>(__builtin_amdgcn_readfirstlane(q));
}

// The experts in the order of their rows, most first, and the places of a tile's outputs.
template <int H, int NT>
struct WeightOrder {
    ExpertRows range;
    int place;                            // lane e: experts in front of expert e
    unsigned row_tiles, col_tiles, tiles; // of an expert: rows, columns, in all
    float per_band;                       // 1 / tiles of four rows

    __device__ __forceinline__ void begin(const WeightTiles& p)
    {
        range = expert_rows(p.offsets, p.E_local, p.max_rows);
        row_tiles = static_cast<unsigned>((p.N + H - 1) / H), col_tiles = static_cast<unsigned>((p.K + NT - 1) / NT);
        tiles = row_tiles * col_tiles;
        per_band = 1.0f / static_cast<float>(kGroupRows * col_tiles);
        const int lane = lane_id(), count = range.hi - range.lo;
        place = lane < p.E_local ? 0 : kWave;
        for (int j = 0; j < p.E_local; ++j) {
            const int other = wave_read_lane(count, j);
            place += other > count || (other == count && j < lane) ? 1 : 0;
        }
    }
    __device__ __forceinline__ int expert(unsigned rank) const { return __builtin_ctzll(__ballot(place == static_cast<int>(rank))); }
    // Four rows of tiles, column by column.
    __device__ __forceinline__ void outputs(unsigned tile, int& row0, int& col0) const
    {
        const unsigned band = quotient(tile, kGroupRows * col_tiles, per_band), in_band = tile - band * kGroupRows * col_tiles;
        const unsigned band_rows = min(static_cast<unsigned>(kGroupRows), row_tiles - band * kGroupRows);
        const unsigned col = band_rows == 3u ? in_band / 3u : in_band >> (band_rows >> 1);
        row0 = __builtin_amdgcn_readfirstlane(static_cast<int>(band * kGroupRows + in_band - col * band_rows) * H);
        col0 = __builtin_amdgcn_readfirstlane(static_cast<int>(col) * NT);
    }
};
constexpr unsigned kMostTiles = 1u << 24;

// A workgroup a tile.
template <int H, int NT, typename TO>
__global__ __launch_bounds__(kProductWaves * kWave, 1) void weight_tiles_kernel(const WeightTiles p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    WeightOrder<H, NT> order;
    order.begin(p);
    const unsigned index = (blockIdx.x / kXcdCount / kGroupTiles * kXcdCount + blockIdx.x % kXcdCount) * kGroupTiles + blockIdx.x / kXcdCount % kGroupTiles;
    const unsigned splits = static_cast<unsigned>(p.splits), part = uniform_udiv(index, order.tiles), rank = uniform_udiv(part, splits), split = part - rank * splits;
    if (rank >= static_cast<unsigned>(p.E_local)) return;
    const int e = order.expert(rank), lo = wave_read_lane(order.range.lo, e), n = wave_read_lane(order.range.hi, e) - lo, stages = (n + 63) / 64;
    int row0, col0;
    order.outputs(index - part * order.tiles, row0, col0);
    const int first = static_cast<int>(static_cast<int64_t>(stages) * split / splits), last = static_cast<int>(static_cast<int64_t>(stages) * (split + 1) / splits);
    const int rows = min(H, p.N - row0), cols = min(NT, p.K - col0);
    const int64_t N = p.N, K = p.K, begin = lo + first * 64, result = (static_cast<int64_t>(split) * p.E_local + e) * N + row0;
    const bool sums = p.sums != nullptr && col0 == 0;
    ProductTile<H, NT, kWeightGradient> t;
    begin_tile(t, smem);
    if (last > first) {
        const int depth = min(n, last * 64) - first * 64;
        t.a.begin(p.dy + begin * N + row0, N * 2, rows, depth, 0, t.wave);
        t.w.begin(p.x + begin * K + col0, K * 2, cols, depth, 0, t.wave);
        t.reduce(last - first, sums);
    } else {
        t.clear();
    }
    if (sums) t.store_sums(static_cast<TO*>(p.sums) + result, rows);
    t.store(static_cast<TO*>(p.out) + result * K + col0, K, rows, cols);
}

// A stream of tiles, not split; PER_UNIT workgroups a compute unit.  What the loads know of a tile goes to the multiplication through a queue in the lanes of a few registers.
template <int H, int NT, int STAGES, int STEPS, int PER_UNIT, bool SUMS, typename TO>
__global__ __launch_bounds__(kProductWaves * kWave, PER_UNIT) void weight_stream_kernel(const WeightTiles p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    typedef ProductTile<H, NT, kWeightGradient, false, STAGES, STEPS> T;
    constexpr int DEPTH = 32 * STEPS;  // rows a stage
    constexpr int STORES = T::template stores<TO>();
    static_assert(T::SA == T::SB, "both operands are loaded of the same stage");
    const int64_t N = p.N, K = p.K;
    WeightOrder<H, NT> order;
    order.begin(p);
    const unsigned step_rank = uniform_udiv(gridDim.x, order.tiles), step_tile = gridDim.x - step_rank * order.tiles;
    const unsigned index = blockIdx.x % kXcdCount * (gridDim.x / kXcdCount) + blockIdx.x / kXcdCount, experts = static_cast<unsigned>(p.E_local);
    unsigned rank = uniform_udiv(index, order.tiles), tile = index - rank * order.tiles;
    int queue_stages = 0, queue_expert = 0, queue_row = 0, queue_col = 0;
    unsigned in = 0u, out = 0u;  // tiles that have entered it and left
    T t;
    begin_tile(t, smem);
    // The next tile with rows is loaded from here on (those without are behind all others); false: there is none.
    auto enter = [&]() {
        if (rank >= experts) return false;
        const int e = order.expert(rank), lo = wave_read_lane(order.range.lo, e), n = wave_read_lane(order.range.hi, e) - lo;
        if (n == 0) return false;
        int row0, col0;
        order.outputs(tile, row0, col0);
        const int64_t begin = lo;
        t.a.begin(p.dy + begin * N + row0, N * 2, min(H, p.N - row0), n, 0, t.wave);
        t.w.begin(p.x + begin * K + col0, K * 2, min(NT, p.K - col0), n, 0, t.wave);
        const bool mine = lane_id() == static_cast<int>(in % kWave);
        queue_stages = mine ? (n + DEPTH - 1) / DEPTH : queue_stages;
        queue_expert = mine ? e : queue_expert;
        queue_row = mine ? row0 : queue_row;
        queue_col = mine ? col0 : queue_col;
        ++in;
        rank += step_rank, tile += step_tile;
        if (tile >= order.tiles) tile -= order.tiles, rank += 1u;
        return true;
    };
    auto feed = [&](T&) {
        if (t.a.todo > 1) {
            t.a.advance();
            t.w.advance();
        } else if (!enter()) {
            t.a.nothing();
            t.w.nothing();
        }
    };
    auto store = [&](int e, int row0, int col0) {
        const int rows = min(H, p.N - row0), cols = min(NT, p.K - col0);
        const int64_t result = e * N + row0;
        if (SUMS && col0 == 0) t.store_sums(static_cast<TO*>(p.sums) + result, rows);
        t.store(static_cast<TO*>(p.out) + result * K + col0, K, rows, cols);
        return rows == H && cols == NT ? 1u : 0u;
    };
    if (enter()) t.template begin_ring<true>(feed, [](T&) {}, []() {});
    unsigned ends = 0u;
    for (; out != in; ++out) {
        const int stages = wave_read_lane(queue_stages, out % kWave), e = wave_read_lane(queue_expert, out % kWave);
        const int row0 = wave_read_lane(queue_row, out % kWave), col0 = wave_read_lane(queue_col, out % kWave);
        t.clear();
        for (int kt = 0; kt < stages; ++kt) {
            t.template stage<true, true, STORES, SUMS>(ends, col0 == 0, feed);
            t.next_stage();
            ends <<= 1;
        }
        t.pin_accumulators();
        ends |= store(e, row0, col0);  // (fewer outputs are fewer stores: those are not counted on)
    }
    wait_vmcnt<0>();  // (loads into LDS that nobody waited for)
    t.clear();
    while (rank < experts) {
        int row0, col0;
        order.outputs(tile, row0, col0);
        store(order.expert(rank), row0, col0);
        rank += step_rank, tile += step_tile;
        if (tile >= order.tiles) tile -= order.tiles, rank += 1u;
    }
}

static int64_t tiles_in(int64_t n, int64_t k, int64_t size) { return ((n + size - 1) / size) * ((k + size - 1) / size); }

// Large tiles where they fill the compute units twice and their reductions are long enough to be worth it.  32 experts of 2048 x 1024, us as large tiles and
// as a stream of small ones: 128 rows an expert 54.5 and 49.0, 200 61.1 and 57.4, 256 65.9 and 64.8, 512 98.7 and 119.3 (results in fp32 76.5 and 62.7, 83.6 and
// 74.4, 87.5 and 82.8, 121.3 and 151.2).
static bool large_tiles(int64_t A, int n, int k, int E_local)
{
    return E_local * tiles_in(n, k, 256) >= 2 * kComputeUnits && A >= 256 * E_local;
}

// Parts of at least 512 rows, at most 16.  Results in fp32, us, with parts of 256, 512 and 1024 rows: 4096 rows, one expert of 512 x 512 21.0, 17.3, 18.9; 2 of
// 1024 x 512 28.6, 20.3, 20.6; 16384 rows, 8 of 256 x 256 20.9, 17.9, 19.2; 1024 rows, one of 512 x 512 12.6, 12.9, 16.3 (not split 16.6).  With at most 8, 16 and 32
// parts: 16384 rows, one of 512 x 512 31.3, 24.7, 36.6, 65536 rows 85, 53, 64 (not split 705); one of 256 x 256 88, 52, 42.
//   As many parts as fill the compute units twice are not always best: 16384 rows, 2 of 1024 x 512 38 in 8 parts and 31 in 4, 65536, 8 of 256 x 256 33 in 16, 23 in 8.
constexpr int kMostSplits = 16;
constexpr int64_t kRowsOfAPart = 512;
int weight_gradient_splits(int64_t A, int n, int k, int E_local)
{
    if (large_tiles(A, n, k, E_local)) return 1;
    const int64_t wanted = 2 * kComputeUnits / (E_local * tiles_in(n, k, 128)), most = A / (E_local * kRowsOfAPart);
    const int64_t s = wanted < most ? wanted : most;
    return static_cast<int>(s < 2 ? 1 : (s > kMostSplits ? kMostSplits : s));
}

static int launch_weight_kernel(void (*kern)(WeightTiles), int64_t grid, size_t lds, std::atomic<uint64_t>& allowed, const WeightTiles& p, hipStream_t stream)
{
    if (int rc = allow_lds(reinterpret_cast<const void*>(kern), lds, allowed, "moe_grouped_product_dw")) return rc;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(kProductWaves * kWave), lds, stream, p);
    return EXF_OK;
}
static int64_t tiles_of(const WeightTiles& p, int H, int NT) { return static_cast<int64_t>((p.N + H - 1) / H) * ((p.K + NT - 1) / NT); }

template <int H, int NT, typename TO>
static int launch_weight_as(const WeightTiles& p, hipStream_t stream)
{
    const int64_t tiles = tiles_of(p, H, NT), groups = (tiles * p.E_local * p.splits + kGroupTiles - 1) / kGroupTiles;
    const int64_t grid = (groups + kXcdCount - 1) / kXcdCount * kXcdCount * kGroupTiles;
    if (tiles >= kMostTiles || grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_dw: too many tiles");
    static std::atomic<uint64_t> allowed{0};
    return launch_weight_kernel(weight_tiles_kernel<H, NT, TO>, grid, product_ring_bytes(H, NT, 128), allowed, p, stream);
}
template <int H, int NT, int STAGES, int STEPS, int PER_UNIT, typename TO>
static int launch_weight_stream(const WeightTiles& p, hipStream_t stream)
{
    constexpr size_t lds = product_ring_bytes(H, NT, 64 * STEPS, STAGES);
    if (tiles_of(p, H, NT) >= kMostTiles) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_dw: too many tiles");
    static std::atomic<uint64_t> allowed{0}, allowed_sums{0};
    if (p.sums != nullptr) return launch_weight_kernel(weight_stream_kernel<H, NT, STAGES, STEPS, PER_UNIT, true, TO>, PER_UNIT * kComputeUnits, lds, allowed_sums, p, stream);
    return launch_weight_kernel(weight_stream_kernel<H, NT, STAGES, STEPS, PER_UNIT, false, TO>, PER_UNIT * kComputeUnits, lds, allowed, p, stream);
}

template <typename TO>
static int launch_weight_tiles(const WeightGradient& g, hipStream_t stream)
{
    const int splits = weight_gradient_splits(g.max_rows, g.N, g.K, g.E_local);
    float* parts = static_cast<float*>(g.workspace);
    const int64_t each = static_cast<int64_t>(g.E_local) * g.N * g.K, sums = static_cast<int64_t>(g.E_local) * g.N;
    WeightTiles p{static_cast<const bf16_t*>(g.dy), static_cast<const bf16_t*>(g.x), g.offsets, g.dw, g.db, g.max_rows, g.N, g.K, g.E_local, splits};
    if (large_tiles(g.max_rows, g.N, g.K, g.E_local)) return launch_weight_as<256, 256, TO>(p, stream);
    if (splits == 1) {
        // Stages of 32 rows, four in a ring, or of 64, two: the same, us: 16 rows an expert 29.8 and 32.5, 32 31.9 and 35.4, 64 36.8 and 37.2, 128 49.0 and
        // 49.5, 200 60.8 and 57.4, 256 69.8 and 64.8.  (One workgroup a compute unit with a ring twice as deep: 42.7, 42.9, 48.1, 59.7, 72.9, 82.4.)
        if (g.max_rows <= 128ll * g.E_local) return launch_weight_stream<128, 128, 4, 1, 2, TO>(p, stream);
        return launch_weight_stream<128, 128, 2, 2, 2, TO>(p, stream);
    }
    p.out = parts;
    if (p.sums != nullptr) p.sums = parts + splits * each;
    if (int rc = launch_weight_as<128, 128, float>(p, stream)) return rc;
    return launch_join_parts(parts, each, g.dw, parts + splits * each, g.db != nullptr ? sums : 0, g.db, splits, sizeof(TO) == 4 ? EXF_F32 : EXF_BF16, stream);
}

int launch_weight_gradient_tiles(const WeightGradient& p, int grad_dt, hipStream_t stream)
{
    return grad_dt == EXF_F32 ? launch_weight_tiles<float>(p, stream) : launch_weight_tiles<bf16_t>(p, stream);
}

}  // namespace exf
