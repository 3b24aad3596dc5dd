// moe_adapters, moe_adapters_backward: low-rank adapters beside a projection that many requests (or an expert's rows) share.
//
//   v_r = A_e x_t,  y_r += s_e B_e^T v_r                                        (row r of adapter e, of token t = perm_src[r] / k)
//   u_r = s_e B_e dy_r,  dx_r = A_e^T u_r,  dA_e = sum_r u_r x_t^T,  dB_e = s_e sum_r v_r dy_r^T
//
// Both matrices lie by rank, [rank, K] and [rank, N], so that the way from dy to dx is the way from x to y with the matrices exchanged: one kernel (moe_adapters_kernel.h), which keeps
// the coefficients v or u on chip between its two products and leaves them in fp32 for the backward pass and the gradients of the matrices (moe_adapters_outer.hip).
#include "moe_adapters.h"

namespace moe {

struct AdapterCall {
    const char *what;
    int dtype, other_dtype, T, k, R, E, K, N, rank, by_assignment;
    const int32_t *perm_src, *offsets;
    const void *a, *b;
};

static int check_adapters(const AdapterCall &c)
{
    const char *what = c.what;
    if (c.T < 0 || c.R < 0 || c.k <= 0 || c.E <= 0) return fail(MOE_ERR_INVALID_ARG, "%s: need T, R >= 0 and k, E > 0", what);
    if (c.K <= 0 || c.N <= 0 || c.K % 8 || c.N % 8) return fail(MOE_ERR_INVALID_ARG, "%s: K and N must be positive multiples of 8 (K=%d N=%d)", what, c.K, c.N);
    if (c.rank <= 0) return fail(MOE_ERR_INVALID_ARG, "%s: rank > 0 required", what);
    if (c.rank > kAdapterMostRank) return fail(MOE_ERR_UNSUPPORTED, "%s: rank %d above %d", what, c.rank, kAdapterMostRank);
    if (c.E > kAdapterMostAdapters) return fail(MOE_ERR_UNSUPPORTED, "%s: %d adapters, above %d", what, c.E, kAdapterMostAdapters);
    if (c.K > 1 << 20 || c.N > 1 << 20) return fail(MOE_ERR_UNSUPPORTED, "%s: K and N of at most 2^20", what);
    if (c.R > kAdapterMostRows) return fail(MOE_ERR_UNSUPPORTED, "%s: %d rows, above %d", what, c.R, kAdapterMostRows);
    if (c.dtype != MOE_F16 && c.dtype != MOE_BF16) return fail(MOE_ERR_UNSUPPORTED, "%s: x and the adapters must be fp16 or bf16", what);
    if (!known_dtype(c.other_dtype)) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (c.R > 0 && !c.perm_src && c.by_assignment) return fail(MOE_ERR_INVALID_ARG, "%s: rows by assignment need perm_src", what);
    if (c.R > 0 && !c.perm_src && c.k != 1) return fail(MOE_ERR_INVALID_ARG, "%s: without perm_src there is one row per row of x (k=%d)", what, c.k);
    if (c.R > 0 && (c.perm_src ? (long long)c.T * c.k != c.R : c.T < c.R)) return fail(MOE_ERR_INVALID_ARG, "%s: %d rows do not fit %d tokens, %d each", what, c.R, c.T, c.k);
    if (!c.offsets || !c.a || !c.b) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(c.a) || !aligned16(c.b)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    return MOE_OK;
}

static int check_rows(const char *what, const char *name, const void *p, int64_t stride, int C)
{
    if (stride < C || stride % 8) return fail(MOE_ERR_INVALID_ARG, "%s: rows of %s must be a multiple of 8 values apart and not overlap", what, name);
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    return MOE_OK;
}

// Rows of a wavefront's part of a matrix's gradient.  Enough parts to fill the chip (a part is 64 channels of `chunk` rows; two thousand wavefronts), as the sums of parts have to be
// written and added up by a launch of their own; at most 1024 rows, or an adapter that has much of the batch is one long chain, unless that would make more than 256 parts of it.  Up to
// 1024 rows, 256 for an adapter on average, are one part, without that launch: 1024 rows of 256 x 256 by 16 adapters take a call of 22.0 us, 24.5 with it.  Of a batch in which one adapter has all the
// rows that is the slower one, which the host cannot see but where there are few adapters (1024 of 1024 x 1024 in one adapter: 31.9 us as one part, 24.5 in parts of 256).
// More rows (a call in parts of 256, 512, 1024, 2048): 16384 by 64 adapters of 4096 x 4096 167, 156, 155, 154 us, 16384 by two 150, 146, 142, 158; 4096 by eight of 1024 x 1024 24.9, 31.2, 31.2.
static int outer_chunk(int R, int C, int E)
{
    if (R <= 1024 && R / 256 <= E) return 1024;
    const long even = (long)R * ((C + 63) / 64) / 2048, most = R / 256 > 1024 ? R / 256 : 1024;
    const long rows = even < 256 ? 256 : even > most ? most : even;
    return (int)((rows + 31) / 32 * 32);
}

static int part_slots(int R, int C, int E) { return 2 * (R / outer_chunk(R, C, E)); }        // n rows in more than one chunk are at most 2 (n / chunk) of them
static size_t part_bytes(int R, int C, int E, int rank) { return (size_t)part_slots(R, C, E) * rank * C * sizeof(float); }

}  // namespace moe

extern "C" int moe_adapters(const void *x, int dtype, int64_t x_stride, int T, const int32_t *perm_src, int k, const int32_t *expert_offsets, int R, int E, int K, int N, int rank,
                            const void *a, const void *b, const float *scale, int by_assignment, const void *y, int64_t y_stride, void *out, int64_t out_stride, int y_dtype, float *v,
                            void *stream)
{
    using namespace moe;
    const char *what = "moe_adapters";
    const AdapterCall call{what, dtype, y_dtype, T, k, R, E, K, N, rank, by_assignment, perm_src, expert_offsets, a, b};
    if (const int rc = check_adapters(call)) return rc;
    if (R == 0) return MOE_OK;                                      // empty buffers may be NULL
    if (!x || !out || (!v && R > kAdapterRowsWithoutV)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(v)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    if (const int rc = check_rows(what, "x", x, x_stride, K)) return rc;
    if (const int rc = check_rows(what, "out", out, out_stride, N)) return rc;
    if (y)
        if (const int rc = check_rows(what, "y", y, y_stride, N)) return rc;
    if (y == out && y_stride != out_stride) return fail(MOE_ERR_INVALID_ARG, "%s: in place the strides of y and out are one", what);
    if (out == x) return fail(MOE_ERR_INVALID_ARG, "%s: out is x, which other blocks still read", what);
    AdapterArgs p{};
    p.offsets = expert_offsets, p.scale = scale, p.R = R, p.E = E, p.K = K, p.N = N, p.rank = rank;
    p.x = x, p.a = a, p.b = b, p.x_map = RowMap{perm_src, k, T, x_stride};
    p.y = y, p.y_stride = y_stride, p.out = out, p.out_map = RowMap{by_assignment ? perm_src : nullptr, 1, R, out_stride};
    p.coef = v, p.coef_scaled = 0;
    return dtype == MOE_F16 ? launch_adapter_forward_f16(p, y_dtype, as_stream(stream), what) : launch_adapter_forward_bf16(p, y_dtype, as_stream(stream), what);
}

extern "C" size_t moe_adapters_backward_workspace_bytes(int R, int E, int K, int N, int rank)
{
    using namespace moe;
    if (R <= 0 || E <= 0 || K <= 0 || N <= 0 || rank <= 0) return 0;
    return round_up((size_t)R * rank * sizeof(float), 256) + round_up(part_bytes(R, K, E, rank), 256) + part_bytes(R, N, E, rank);
}

extern "C" int moe_adapters_backward(const void *dy, int dy_dtype, int64_t dy_stride, const void *x, int dtype, int64_t x_stride, int T, const int32_t *perm_src, int k,
                                     const int32_t *expert_offsets, int R, int E, int K, int N, int rank, const void *a, const void *b, const float *scale, int by_assignment,
                                     const float *v, void *dx, int64_t dx_stride, void *da, void *db, int grad_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace moe;
    const char *what = "moe_adapters_backward";
    const AdapterCall call{what, dtype, dy_dtype, T, k, R, E, K, N, rank, by_assignment, perm_src, expert_offsets, a, b};
    if (const int rc = check_adapters(call)) return rc;
    if (!known_dtype(grad_dtype)) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (!aligned16(da) || !aligned16(db)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    if (R > 0) {
        if (!dy || (da && !x) || (db && !v)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
        if (const int rc = check_rows(what, "dy", dy, dy_stride, N)) return rc;
        if (da)
            if (const int rc = check_rows(what, "x", x, x_stride, K)) return rc;
        if (dx)
            if (const int rc = check_rows(what, "dx", dx, dx_stride, K)) return rc;
        const size_t need = moe_adapters_backward_workspace_bytes(R, E, K, N, rank);
        if (!workspace || workspace_bytes < need) return fail(MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", what, need, workspace_bytes);
        if (!aligned16(workspace) || !aligned16(v)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
        if (dx && (dx == dy || dx == x)) return fail(MOE_ERR_INVALID_ARG, "%s: dx is dy or x, which are still read", what);
    }
    const hipStream_t s = as_stream(stream);
    const RowMap tokens{perm_src, k, T, x_stride}, rows{by_assignment ? perm_src : nullptr, 1, R, dy_stride};
    float *u = (float *)workspace, *part0 = R > 0 ? (float *)((char *)workspace + round_up((size_t)R * rank * sizeof(float), 256)) : nullptr;
    float *part1 = R > 0 ? (float *)((char *)part0 + round_up(part_bytes(R, K, E, rank), 256)) : nullptr;
    if (R > 0 && (dx || da)) {
        AdapterArgs p{};
        p.offsets = expert_offsets, p.scale = scale, p.R = R, p.E = E, p.K = N, p.N = K, p.rank = rank;
        p.x = dy, p.a = b, p.b = a, p.x_map = rows;
        p.out = dx, p.out_map = RowMap{rows.source, 1, R, dx_stride};
        p.coef = u, p.coef_scaled = 1;
        const int rc = dtype == MOE_F16 ? launch_adapter_backward_f16(p, dy_dtype, s, what) : launch_adapter_backward_bf16(p, dy_dtype, s, what);
        if (rc != MOE_OK) return rc;
    }
    OuterArgs p{};
    p.offsets = expert_offsets, p.R = R, p.E = E, p.rank = rank, p.out_dtype = grad_dtype;
    p.job[0] = OuterJob{x, tokens, u, nullptr, da, K, 0, outer_chunk(R, K, E), part0, part_slots(R, K, E)};
    p.job[1] = OuterJob{dy, rows, v, scale, db, N, 0, outer_chunk(R, N, E), part1, part_slots(R, N, E)};
    return launch_adapter_outer(p, dtype, dy_dtype, s, what);
}
