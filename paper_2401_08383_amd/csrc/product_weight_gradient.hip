// Weight gradient of the experts' products in tiles, bf16 (see product_tiles.hpp): dw[e][N,K] = dy[rows of e, N]^T x[rows of e, K].
//
// The reduction is an expert's rows, so its length differs from expert to expert and all tiles of an expert take equally long:
// the longest experts come first.  Tiles go out in groups of 32, as many as an XCD has compute units: four rows of tiles by eight
// columns, which share their operands in that XCD's L2.
//   Few tiles: the reduction is split, the parts' sums go to the workspace in fp32, and a second launch adds them up in order.
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

template <int H, int NT, int STAGES, typename TO>
__global__ __launch_bounds__(kProductWaves * kWave, STAGES == 2 ? 2 : 1) void weight_tiles_kernel(const WeightTiles p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const RowRange range = row_range(p.offsets, p.E_local, p.max_rows);
    const int lane = lane_id(), count = range.hi - range.lo;
    const unsigned row_tiles = static_cast<unsigned>((p.N + H - 1) / H), col_tiles = static_cast<unsigned>((p.K + NT - 1) / NT), tiles = row_tiles * col_tiles;
    const unsigned groups = (tiles + kGroupTiles - 1) / kGroupTiles;  // of an expert's part
    const unsigned xcd = blockIdx.x % kXcdCount, pos = blockIdx.x / kXcdCount;
    const unsigned group = pos / kGroupTiles * kXcdCount + xcd;
    const unsigned part = uniform_udiv(group, groups), tile = (group - part * groups) * kGroupTiles + pos % kGroupTiles;
    const unsigned rank = uniform_udiv(part, static_cast<unsigned>(p.splits)), split = part - rank * static_cast<unsigned>(p.splits);
    if (rank >= static_cast<unsigned>(p.E_local) || tile >= tiles) return;
    int longer = 0;  // experts in front of expert `lane`
    for (int j = 0; j < p.E_local; ++j) {
        const int other = wave_read_lane(count, j);
        longer += other > count || (other == count && j < lane) ? 1 : 0;
    }
    const int e = __builtin_ctzll(__ballot(lane < p.E_local && longer == static_cast<int>(rank)));
    const int lo = wave_read_lane(range.lo, e), n = wave_read_lane(count, e);
    // four rows of tiles, column by column
    const unsigned band = uniform_udiv(tile, kGroupRows * col_tiles), in_band = tile - band * kGroupRows * col_tiles;
    const unsigned band_rows = min(static_cast<unsigned>(kGroupRows), row_tiles - band * kGroupRows);
    const unsigned col_tile = uniform_udiv(in_band, band_rows);
    const int row0 = __builtin_amdgcn_readfirstlane(static_cast<int>(band * kGroupRows + in_band - col_tile * band_rows)) * H;
    const int col0 = __builtin_amdgcn_readfirstlane(static_cast<int>(col_tile)) * NT;

    const int stages = (n + 63) / 64;
    const int first = static_cast<int>(static_cast<int64_t>(stages) * split / p.splits), last = static_cast<int>(static_cast<int64_t>(stages) * (split + 1) / p.splits);
    const int rows = min(n, last * 64) - first * 64;
    const int64_t begin = lo + first * 64, N = p.N, K = p.K;
    ProductTile<H, NT, kWeightGradient, false, STAGES> t;
    begin_tile(t, smem);
    const bool sums = p.sums != nullptr && col0 == 0;
    if (rows > 0) {
        t.a.begin(p.dy + begin * N + row0, N * 2, min(H, p.N - row0), rows, 0, t.wave);
        t.w.begin(p.x + begin * K + col0, K * 2, min(NT, p.K - col0), rows, 0, t.wave);
        if (sums) t.template reduce<true>(last - first);
        else t.reduce(last - first);
    } else {
        t.clear();
    }
    if (sums) t.store_sums(static_cast<TO*>(p.sums) + (static_cast<int64_t>(split) * p.E_local + e) * N + row0, min(H, p.N - row0));
    t.store(static_cast<TO*>(p.out) + ((static_cast<int64_t>(split) * p.E_local + e) * N + row0) * K + col0, K, min(H, p.N - row0), min(NT, p.K - col0), nullptr);
}

static int64_t tiles_in(int64_t n, int64_t k, int64_t size) { return ((n + size - 1) / size) * ((k + size - 1) / size); }

// Large tiles where they fill the compute units twice and their reductions are long enough to be worth it.
static bool large_tiles(int64_t A, int n, int k, int E_local)
{
    return E_local * tiles_in(n, k, 256) >= 2 * kComputeUnits && A >= 256 * E_local;
}

constexpr int kMostSplits = 16;
constexpr int64_t kRowsOfAPart = 512;
int weight_gradient_splits(int64_t A, int n, int k, int E_local)
{
    if (large_tiles(A, n, k, E_local)) return 1;
    const int64_t wanted = 2 * kComputeUnits / (E_local * tiles_in(n, k, 128)), most = A / (E_local * kRowsOfAPart);
    const int64_t s = wanted < most ? wanted : most;
    return static_cast<int>(s < 2 ? 1 : (s > kMostSplits ? kMostSplits : s));
}

template <int H, int NT, int STAGES, typename TO>
static int launch_weight_as(const WeightTiles& p, hipStream_t stream)
{
    constexpr size_t lds = product_ring_bytes(H, NT, 128, STAGES);
    const int64_t tiles = static_cast<int64_t>((p.N + H - 1) / H) * ((p.K + NT - 1) / NT);
    const int64_t groups = (tiles + kGroupTiles - 1) / kGroupTiles * p.E_local * p.splits;
    const int64_t grid = (groups + kXcdCount - 1) / kXcdCount * kXcdCount * kGroupTiles;
    if (tiles >= (1ll << 31) || grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "moe_grouped_product_dw: too many tiles");
    auto kern = weight_tiles_kernel<H, NT, STAGES, TO>;
    static std::atomic<uint64_t> allowed{0};
    if (int rc = allow_lds(reinterpret_cast<const void*>(kern), lds, allowed, "moe_grouped_product_dw")) return rc;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(kProductWaves * kWave), lds, stream, p);
    return EXF_OK;
}

template <typename TO>
static int launch_weight_tiles(const WeightGradient& g, hipStream_t stream)
{
    const int splits = weight_gradient_splits(g.max_rows, g.N, g.K, g.E_local);
    float* parts = static_cast<float*>(g.workspace);
    const int64_t each = static_cast<int64_t>(g.E_local) * g.N * g.K, sums = static_cast<int64_t>(g.E_local) * g.N;
    WeightTiles p{static_cast<const bf16_t*>(g.dy), static_cast<const bf16_t*>(g.x), g.offsets, g.dw, g.db, g.max_rows, g.N, g.K, g.E_local, splits};
    if (large_tiles(g.max_rows, g.N, g.K, g.E_local)) return launch_weight_as<256, 256, 8, TO>(p, stream);
    if (splits == 1) return launch_weight_as<128, 128, 2, TO>(p, stream);
    p.out = parts;
    if (p.sums != nullptr) p.sums = parts + splits * each;
    if (int rc = launch_weight_as<128, 128, 2, float>(p, stream)) return rc;
    return launch_join_parts(parts, each, g.dw, parts + splits * each, g.db != nullptr ? sums : 0, g.db, splits, sizeof(TO) == 4 ? EXF_F32 : EXF_BF16, stream);
}

int launch_weight_gradient_tiles(const WeightGradient& p, int grad_dt, hipStream_t stream)
{
    return grad_dt == EXF_F32 ? launch_weight_tiles<float>(p, stream) : launch_weight_tiles<bf16_t>(p, stream);
}

}  // namespace exf
