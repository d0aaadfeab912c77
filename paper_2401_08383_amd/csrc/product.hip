// Entry points of the experts' products: checks, and the choice of kernels.
#include "product_tiles.hpp"

namespace exf {

int check_product_sizes(const char* fn, int64_t A, int n, int k, int E_local, int dt)
{
    if (dt != EXF_F32 && dt != EXF_BF16) return fail(EXF_ERR_BAD_DTYPE, "%s: dt = %d", fn, dt);
    if (A < 0 || A > EXF_MAX_PRODUCT_ROWS) return fail(EXF_ERR_BAD_SHAPE, "%s: A = %lld outside [0,%lld]", fn, static_cast<long long>(A), EXF_MAX_PRODUCT_ROWS);
    if (E_local < 1 || E_local > EXF_MAX_EXPERTS) return fail(EXF_ERR_BAD_SHAPE, "%s: E_local = %d outside [1,%d]", fn, E_local, EXF_MAX_EXPERTS);
    const int gran = dt == EXF_BF16 ? 8 : 4;
    if (n < gran || n % gran != 0 || k < gran || k % gran != 0)
        return fail(EXF_ERR_BAD_SHAPE, "%s: n = %d and k = %d must be positive multiples of %d", fn, n, k, gran);
    if (n > EXF_MAX_PRODUCT_WIDTH || k > EXF_MAX_PRODUCT_WIDTH)  // the tiles address their rows with 32-bit byte offsets
        return fail(EXF_ERR_BAD_SHAPE, "%s: n = %d and k = %d must not exceed %d", fn, n, k, EXF_MAX_PRODUCT_WIDTH);
    return EXF_OK;
}

static size_t type_bytes(int dt) { return dt == EXF_BF16 ? 2 : 4; }

static int check_rows_product(const char* fn, const void* rows, const int32_t* offsets, const void* w, const void* bias, int64_t A, int n, int k,
                              int E_local, int dt, bool gradient, const void* out)
{
    if (int rc = check_product_sizes(fn, A, n, k, E_local, dt)) return rc;
    if (A == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, rows);
    EXF_CHECK_PTR(fn, offsets);
    EXF_CHECK_PTR(fn, w);
    EXF_CHECK_PTR(fn, out);
    EXF_CHECK_ALIGNED(fn, rows);
    EXF_CHECK_ALIGNED(fn, w);
    EXF_CHECK_ALIGNED(fn, out);
    if (bias != nullptr) EXF_CHECK_ALIGNED(fn, bias);
    const size_t el = type_bytes(dt), in = static_cast<size_t>(A) * (gradient ? n : k) * el, o = static_cast<size_t>(A) * (gradient ? k : n) * el;
    if (overlap(out, o, rows, in) || overlap(out, o, w, static_cast<size_t>(E_local) * n * k * el) || overlap(out, o, bias, static_cast<size_t>(E_local) * n * el) ||
        overlap(out, o, offsets, static_cast<size_t>(E_local + 1) * 4))
        return fail(EXF_ERR_BAD_SHAPE, "%s: the result must not overlap an input", fn);
    return EXF_OK;
}

// Few rows an expert: a stream of weights (ffn_stream.hip), in its sizes.  Tiles and streams, us, rows spread evenly: 64 experts of 4096 x 1024 with 16 rows
// each 87 and 82, 24 89 and 89, 28 90 and 92, 48 91 and 113; 64 of 1024 x 4096 24 84 and 82, 48 86 and 93; 8 of 8192 x 2048 16 41 and 42, 28 41 and 43; 8 of
// 4096 x 1024 24 14.2 and 12.0, 48 14.3 and 14.8; 4 of 2048 x 8192 28 41 and 25, 48 41 and 47; 32 of 512 x 512 6.6 and 6.1, with 64 rows 6.8 and 6.2.
//   The rule knows the mean only.  Skewed, 24 rows an expert: 64 of 4096 x 1024, rows as 1/rank 96 and 111, all 1536 on one, whose weights every tile of 64
// rows reads again, 19.6 and 47.4; 8 of 4096 x 1024 15.6 and 15.4, on one 10.0 and 8.4; 16 of 1024 x 1024 12.5 and 10.5, on one 9.8 and 8.2.
static bool streams_forward(int64_t A, int n, int k, int E_local)
{
    const int64_t widest = n > k ? n : k;
    return n % 64 == 0 && k % 64 == 0 && A <= 28ll * E_local && A * widest < (1ll << 31) && static_cast<int64_t>(n) * k < (1ll << 31);
}

// fp32 with more rows an expert, the more the longer the reduction is: tiles (product_exact.hip).  Streams and tiles, us, rows skewed (and even): 8 experts of
// 1024 x 1024, 4096 rows 149 and 95 (79 and 78); 32 of 512 x 512, 16384 rows 130 and 87 (91 and 85); of 24 rows an expert 40 of 1024 x 1024 78 and 60 (47 and 58),
// 20 of 2048 x 256 29 and 18 (17 and 17), 8 of 2048 x 1024 31 and 22 (30 and 22), 4 of 1024 x 4096 31 and 38 (of 48 rows 58 and 39), 2 of 256 x 8192 30 and 72 (96
// rows 31 and 72, 500 rows 114 and 73); of 16 rows 40 of 1024 x 1024 44 and 59 (35 and 59).
static bool exact_forward_in_tiles(int64_t A, int k, int E_local) { return A >= (k <= 2048 ? 24ll : (k <= 4096 ? 48ll : 128ll)) * E_local; }

}  // namespace exf

extern "C" int moe_grouped_product(const void* x_sorted, const int32_t* expert_offsets, const void* w, const void* bias, int64_t A, int n, int k,
                                   int E_local, int dt, void* y_sorted, void* stream)
{
    using namespace exf;
    if (int rc = check_rows_product("moe_grouped_product", x_sorted, expert_offsets, w, bias, A, n, k, E_local, dt, false, y_sorted)) return rc;
    if (A == 0) return EXF_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int rc;
    if (dt == EXF_F32 && exact_forward_in_tiles(A, k, E_local)) {
        rc = launch_exact_product({x_sorted, expert_offsets, w, bias, y_sorted, static_cast<int>(A), k, n, E_local}, s);
    } else if (dt == EXF_F32 || streams_forward(A, n, k, E_local)) {
        StreamGemm g{};
        g.act = x_sorted, g.weight = w, g.bias = bias, g.out = y_sorted, g.offsets = expert_offsets;
        g.max_rows = static_cast<int>(A), g.K = k, g.N = n, g.E_local = E_local, g.epi = kEpiNone;
        rc = launch_stream_gemm(g, dt, s, "moe_grouped_product");
    } else {
        rc = launch_forward_tiles({x_sorted, expert_offsets, w, static_cast<const bf16_t*>(bias), static_cast<bf16_t*>(y_sorted), nullptr, nullptr, static_cast<int>(A), k, n, E_local}, s);
    }
    return rc == EXF_OK ? check_launch("moe_grouped_product") : rc;
}

extern "C" int moe_grouped_product_dx(const void* dy_sorted, const int32_t* expert_offsets, const void* w, int64_t A, int n, int k, int E_local, int dt,
                                      void* dx_sorted, void* stream)
{
    using namespace exf;
    if (int rc = check_rows_product("moe_grouped_product_dx", dy_sorted, expert_offsets, w, nullptr, A, n, k, E_local, dt, true, dx_sorted)) return rc;
    if (A == 0) return EXF_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int rc;
    if (dt == EXF_BF16) {
        rc = launch_rows_gradient_tiles({dy_sorted, expert_offsets, w, nullptr, static_cast<bf16_t*>(dx_sorted), nullptr, nullptr, static_cast<int>(A), n, k, E_local}, s);
    } else {
        rc = launch_exact_rows_gradient({dy_sorted, expert_offsets, w, nullptr, dx_sorted, static_cast<int>(A), n, k, E_local}, s);
    }
    return rc == EXF_OK ? check_launch("moe_grouped_product_dx") : rc;
}

// Sizes that a workspace is computed for: others are refused by the call, and would overflow on the way.
static bool sizes_fit(int64_t A, int n, int k)
{
    return A >= 1 && A <= EXF_MAX_PRODUCT_ROWS && n >= 1 && n <= EXF_MAX_PRODUCT_WIDTH && k >= 1 && k <= EXF_MAX_PRODUCT_WIDTH;
}

extern "C" size_t moe_grouped_product_dw_workspace_bytes(int64_t A, int n, int k, int E_local, int dt)
{
    if (!sizes_fit(A, n, k) || E_local < 1 || E_local > EXF_MAX_EXPERTS || (dt != EXF_BF16 && dt != EXF_F32)) return 0;
    const int splits = dt == EXF_BF16 ? exf::weight_gradient_splits(A, n, k, E_local) : exf::exact_weight_gradient_splits(A, n, k, E_local);
    return splits > 1 ? exf::align_up(static_cast<size_t>(splits) * E_local * n * (static_cast<size_t>(k) + 1) * 4, 256) : 0;  // dw's and db's
}

extern "C" int moe_grouped_product_dw(const void* dy_sorted, const void* x_sorted, const int32_t* expert_offsets, int64_t A, int n, int k, int E_local,
                                      int dt, int grad_dt, void* dw, void* db, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace exf;
    const char* fn = "moe_grouped_product_dw";
    if (int rc = check_product_sizes(fn, A, n, k, E_local, dt)) return rc;
    if (grad_dt != EXF_F32 && grad_dt != dt) return fail(EXF_ERR_BAD_DTYPE, "%s: grad_dt = %d with dt = %d", fn, grad_dt, dt);
    if (A > 0) {
        EXF_CHECK_PTR(fn, dy_sorted);
        EXF_CHECK_PTR(fn, x_sorted);
        EXF_CHECK_ALIGNED(fn, dy_sorted);
        EXF_CHECK_ALIGNED(fn, x_sorted);
    }
    EXF_CHECK_PTR(fn, expert_offsets);
    EXF_CHECK_PTR(fn, dw);
    EXF_CHECK_ALIGNED(fn, dw);
    if (db != nullptr) EXF_CHECK_ALIGNED(fn, db);
    const size_t need = moe_grouped_product_dw_workspace_bytes(A, n, k, E_local, dt);
    if (need > 0) {
        EXF_CHECK_PTR(fn, workspace);
        EXF_CHECK_ALIGNED(fn, workspace);
        if (workspace_bytes < need) return fail(EXF_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < %zu bytes", fn, workspace_bytes, need);
    }
    const size_t el = type_bytes(dt), grad = type_bytes(grad_dt), experts = E_local, rows = A;
    const struct {
        const void* at;
        size_t bytes;
    } in[] = {{dy_sorted, rows * n * el}, {x_sorted, rows * k * el}, {expert_offsets, (experts + 1) * 4}}, out[] = {{dw, experts * n * k * grad}, {db, experts * n * grad}, {workspace, need}};
    for (const auto& o : out)
        for (const auto& i : in)
            if (overlap(o.at, o.bytes, i.at, i.bytes)) return fail(EXF_ERR_BAD_SHAPE, "%s: results and workspace must not overlap an input", fn);
    if (overlap(dw, out[0].bytes, db, out[1].bytes) || overlap(workspace, need, dw, out[0].bytes) || overlap(workspace, need, db, out[1].bytes))
        return fail(EXF_ERR_BAD_SHAPE, "%s: results and workspace must not overlap", fn);
    const WeightGradient p{dy_sorted, x_sorted, expert_offsets, dw, db, workspace, static_cast<int>(A), n, k, E_local};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc = dt == EXF_BF16 ? launch_weight_gradient_tiles(p, grad_dt, s) : launch_exact_weight_gradient(p, s);
    return rc == EXF_OK ? check_launch(fn) : rc;
}

extern "C" size_t moe_grouped_product_mx4_workspace_bytes(int64_t A, int n, int k)
{
    if (!sizes_fit(A, n, k) || exf::mx4_product_is_small(A, n, k)) return 0;
    return exf::align_up(static_cast<size_t>(A) * k / 2, 256) + exf::align_up(mx4_scale_bytes(A, k), 256);
}

extern "C" int moe_grouped_product_mx4(const void* x_sorted, const uint8_t* x_scale, const int32_t* expert_offsets, const uint8_t* w, const uint8_t* w_scale,
                                       const void* bias, int64_t A, int n, int k, int E_local, int dt, void* y_sorted, void* workspace,
                                       size_t workspace_bytes, void* stream)
{
    using namespace exf;
    const char* fn = "moe_grouped_product_mx4";
    if (int rc = check_product_sizes(fn, A, n, k, E_local, dt)) return rc;
    if (k % EXF_MX4_BLOCK != 0) return fail(EXF_ERR_BAD_SHAPE, "%s: k = %d must be a multiple of %d", fn, k, EXF_MX4_BLOCK);
    if (A == 0) return EXF_OK;
    EXF_CHECK_PTR(fn, x_sorted);
    EXF_CHECK_PTR(fn, expert_offsets);
    EXF_CHECK_PTR(fn, w);
    EXF_CHECK_PTR(fn, w_scale);
    EXF_CHECK_PTR(fn, y_sorted);
    EXF_CHECK_ALIGNED(fn, x_sorted);
    EXF_CHECK_ALIGNED(fn, w);
    EXF_CHECK_ALIGNED(fn, w_scale);
    EXF_CHECK_ALIGNED(fn, y_sorted);
    if (x_scale != nullptr) EXF_CHECK_ALIGNED(fn, x_scale);
    if (bias != nullptr) EXF_CHECK_ALIGNED(fn, bias);
    const size_t need = x_scale == nullptr ? moe_grouped_product_mx4_workspace_bytes(A, n, k) : 0;
    if (need > 0) {
        EXF_CHECK_PTR(fn, workspace);
        EXF_CHECK_ALIGNED(fn, workspace);
        if (workspace_bytes < need) return fail(EXF_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < %zu bytes", fn, workspace_bytes, need);
    }
    const size_t el = type_bytes(dt), rows = A, held = rows * k / 2, weights = static_cast<size_t>(E_local) * n, out_bytes = rows * n * el;
    const struct {
        const void* at;
        size_t bytes;
    } in[] = {{x_sorted, x_scale == nullptr ? rows * k * el : held}, {x_scale, mx4_scale_bytes(A, k)}, {expert_offsets, static_cast<size_t>(E_local + 1) * 4},
              {w, weights * k / 2}, {w_scale, mx4_scale_bytes(static_cast<int64_t>(weights), k)}, {bias, weights * el}};
    for (const auto& i : in)
        if (overlap(y_sorted, out_bytes, i.at, i.bytes) || overlap(workspace, need, i.at, i.bytes))
            return fail(EXF_ERR_BAD_SHAPE, "%s: the result and the workspace must not overlap an input", fn);
    if (overlap(workspace, need, y_sorted, out_bytes)) return fail(EXF_ERR_BAD_SHAPE, "%s: the result and the workspace must not overlap", fn);
    Mx4Product p{static_cast<const uint8_t*>(x_sorted), x_scale, expert_offsets, w, w_scale, bias, y_sorted, static_cast<int>(A), k, n, E_local};
    if (need > 0) {
        uint8_t* q = static_cast<uint8_t*>(workspace);
        uint8_t* scale = q + align_up(held, 256);
        if (int rc = mx4_quantize(x_sorted, A, k, dt, q, scale, stream)) return rc;
        p.rows = q, p.row_scale = scale;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    int rc;
    if (mx4_product_is_small(A, n, k)) {
        rc = launch_mx4_small(p, dt, s);
    } else if (dt == EXF_BF16) {
        rc = launch_mx4_tiles({p.rows, expert_offsets, w, static_cast<const bf16_t*>(bias), static_cast<bf16_t*>(y_sorted), p.row_scale, w_scale, static_cast<int>(A), k, n, E_local}, s);
    } else {
        rc = launch_mx4_product(p, s);
    }
    return rc == EXF_OK ? check_launch(fn) : rc;
}
