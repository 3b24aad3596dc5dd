// moe_adapters, moe_adapters_backward: low-rank adapters beside a projection that many requests (or an expert's rows) share.
//
//   v_r = A_e x_t,  y_r += s_e B_e^T v_r                                        (row r of adapter e, of token t = perm_src[r] / k)
//   u_r = s_e B_e dy_r,  dx_r = A_e^T u_r,  dA_e = sum_r u_r x_t^T,  dB_e = s_e sum_r v_r dy_r^T
//
// Both matrices lie by rank, [rank, K] and [rank, N], so that three products make up all of it: rows times a matrix along their channels ("shrink": v, u), coefficients times a matrix
// along the rank ("expand": y, dx), and coefficients times rows along an adapter's rows ("outer": dA, dB).  Coefficients are kept in fp32.
#include "moe_rows.h"

namespace moe {

constexpr int kAdapterMostRank = 128, kAdapterMostAdapters = 4096;

// Where row r of the sorted order is found: in rows of tokens (source / k), of assignments (source), or in place.
struct RowMap {
    const int32_t *source;      // perm_src or null
    int div;                    // k for tokens, 1 for assignments
    int rows;                   // of the buffer
    int64_t stride;

    __device__ inline size_t at(int r) const { return (size_t)(source ? min(max(source[r] / div, 0), rows - 1) : r) * stride; }
};

struct AdapterArgs {
    const int32_t *offsets;     // [E + 1]
    const float *scale;         // [E] or null
    int R, E, C, rank;          // C: channels
    const void *rows;           // shrink, outer: what is multiplied; expand: what the product is added to, or null
    RowMap map;
    const void *w;              // [E, rank, C]
    float *coef;                // [R, rank]: shrink writes it, expand and outer read it
    void *out;                  // expand: rows, by out_map; outer: [E, rank, C]
    RowMap out_map;
};

// Adapter of row r: the last one that begins at or before it; false for rows behind the last adapter's.
__device__ inline bool adapter_of(const AdapterArgs &p, int r, int *e)
{
    int lo = 0, hi = p.E;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (p.offsets[mid] <= r) lo = mid;
        else hi = mid;
    }
    *e = lo;
    return p.offsets[lo] <= r && r < p.offsets[lo + 1];
}

// coef[r][j] = scale <rows[r], w[e][j]>
template <int DT, int WDT>
__global__ __launch_bounds__(256) void adapter_shrink_kernel(AdapterArgs p)
{
    const int r = blockIdx.x, lane = threadIdx.x & 63;
    int e;
    if (!adapter_of(p, r, &e)) return;
    const size_t at = p.map.at(r);
    const float s = p.scale ? p.scale[e] : 1.0f;
    for (int j = threadIdx.x >> 6; j < p.rank; j += 4) {
        const size_t row = ((size_t)e * p.rank + j) * p.C;
        float sum = 0.0f;
        for (int c = lane * 8; c < p.C; c += 512) {
            Raw<DT, 8> x;
            Raw<WDT, 8> w;
            x.load(p.rows, at + c), w.load(p.w, row + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(x.get(i), w.get(i), sum);
        }
        sum = wave_sum(sum);
        if (lane == 0) p.coef[(size_t)r * p.rank + j] = s * sum;
    }
}

// out[r] = rows[r] + scale sum_j coef[r][j] w[e][j]; rows of no adapter are copied where out is another buffer
template <int DT, int WDT>
__global__ __launch_bounds__(256) void adapter_expand_kernel(AdapterArgs p)
{
    const int r = blockIdx.x;
    int e;
    const bool live = adapter_of(p, r, &e);
    if (!live && p.rows == p.out) return;
    const size_t from = p.map.at(r), to = p.out_map.at(r);
    const float s = p.scale ? p.scale[e] : 1.0f;
    for (int c = threadIdx.x * 8; c < p.C; c += 2048) {
        Raw<DT, 8> y;
        if (p.rows) y.load(p.rows, from + c);
        else y.clear();
        if (live) {
            float v[8] = {};
            for (int j = 0; j < p.rank; ++j) {
                const float f = p.coef[(size_t)r * p.rank + j] * s;
                Raw<WDT, 8> w;
                w.load(p.w, ((size_t)e * p.rank + j) * p.C + c);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = fmaf(f, w.get(i), v[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += y.get(i);
            y.set(v);
        }
        y.store(p.out, to + c);
    }
}

// out[e][j] = scale sum_r coef[r][j] rows[r]
template <int DT, int ODT>
__global__ __launch_bounds__(256) void adapter_outer_kernel(AdapterArgs p)
{
    const int e = blockIdx.x, j = blockIdx.y;
    int lo, hi;
    expert_range(p.offsets, e, p.R, &lo, &hi);
    const float s = p.scale ? p.scale[e] : 1.0f;
    for (int c = threadIdx.x * 8; c < p.C; c += 2048) {
        float v[8] = {};
        for (int r = lo; r < hi; ++r) {
            const float f = p.coef[(size_t)r * p.rank + j];
            Raw<DT, 8> x;
            x.load(p.rows, p.map.at(r) + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(f, x.get(i), v[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= s;
        Raw<ODT, 8> o;
        o.set(v);
        o.store(p.out, ((size_t)e * p.rank + j) * p.C + c);
    }
}

static size_t coefficient_bytes(int R, int rank) { return round_up((size_t)R * rank * sizeof(float), 256); }

template <class F>
static int with_half(int dtype, F &&f)
{
    return dtype == MOE_F16 ? f(std::integral_constant<int, MOE_F16>{}) : f(std::integral_constant<int, MOE_BF16>{});
}

static int launch_shrink(const AdapterArgs &p, int dtype, int w_dtype, hipStream_t s, const char *what)
{
    return with_dtype(dtype, [&](auto d) {
        return with_half(w_dtype, [&](auto w) {
            hipLaunchKernelGGL((adapter_shrink_kernel<decltype(d)::value, decltype(w)::value>), dim3(p.R), dim3(256), 0, s, p);
            return check_launch(what);
        });
    });
}

static int launch_expand(const AdapterArgs &p, int dtype, int w_dtype, hipStream_t s, const char *what)
{
    return with_dtype(dtype, [&](auto d) {
        return with_half(w_dtype, [&](auto w) {
            hipLaunchKernelGGL((adapter_expand_kernel<decltype(d)::value, decltype(w)::value>), dim3(p.R), dim3(256), 0, s, p);
            return check_launch(what);
        });
    });
}

static int launch_outer(const AdapterArgs &p, int dtype, int out_dtype, hipStream_t s, const char *what)
{
    return with_dtype(dtype, [&](auto d) {
        return with_dtype(out_dtype, [&](auto o) {
            hipLaunchKernelGGL((adapter_outer_kernel<decltype(d)::value, decltype(o)::value>), dim3(p.E, p.rank), dim3(256), 0, s, p);
            return check_launch(what);
        });
    });
}

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
    if (c.K > 1 << 24 || c.N > 1 << 24) return fail(MOE_ERR_UNSUPPORTED, "%s: K and N of at most 2^24", what);
    if (c.R >= 1 << 24) return fail(MOE_ERR_UNSUPPORTED, "%s: fewer than 2^24 rows", what);
    if (c.dtype != MOE_F16 && c.dtype != MOE_BF16) return fail(MOE_ERR_UNSUPPORTED, "%s: x and the adapters must be fp16 or bf16", what);
    if (!known_dtype(c.other_dtype)) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (!c.perm_src && c.by_assignment) return fail(MOE_ERR_INVALID_ARG, "%s: rows by assignment need perm_src", what);
    if (!c.perm_src && c.k != 1) return fail(MOE_ERR_INVALID_ARG, "%s: without perm_src there is one row per row of x (k=%d)", what, c.k);
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

}  // namespace moe

extern "C" size_t moe_adapters_workspace_bytes(int R, int E, int K, int N, int rank)
{
    if (R <= 0 || E <= 0 || K <= 0 || N <= 0 || rank <= 0) return 0;
    return moe::coefficient_bytes(R, rank);
}

extern "C" int moe_adapters(const void *x, int dtype, int64_t x_stride, int T, const int32_t *perm_src, int k, const int32_t *expert_offsets, int R, int E, int K, int N, int rank,
                            const void *a, const void *b, const float *scale, int by_assignment, const void *y, int64_t y_stride, void *out, int64_t out_stride, int y_dtype, float *v,
                            void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace moe;
    const char *what = "moe_adapters";
    const AdapterCall call{what, dtype, y_dtype, T, k, R, E, K, N, rank, by_assignment, perm_src, expert_offsets, a, b};
    if (const int rc = check_adapters(call)) return rc;
    if (R == 0) return MOE_OK;                                      // empty buffers may be NULL
    if (!x || !out) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (const int rc = check_rows(what, "x", x, x_stride, K)) return rc;
    if (const int rc = check_rows(what, "out", out, out_stride, N)) return rc;
    if (y)
        if (const int rc = check_rows(what, "y", y, y_stride, N)) return rc;
    if (y == out && y_stride != out_stride) return fail(MOE_ERR_INVALID_ARG, "%s: in place the strides of y and out are one", what);
    const size_t need = moe_adapters_workspace_bytes(R, E, K, N, rank);
    if (!workspace || workspace_bytes < need) return fail(MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", what, need, workspace_bytes);
    if (!aligned16(workspace) || !aligned16(v)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const hipStream_t s = as_stream(stream);
    const RowMap tokens{perm_src, k, T, x_stride}, y_map{by_assignment ? perm_src : nullptr, 1, R, y_stride}, out_map{by_assignment ? perm_src : nullptr, 1, R, out_stride};
    float *coef = v ? v : (float *)workspace;
    AdapterArgs p{expert_offsets, nullptr, R, E, K, rank, x, tokens, a, coef, nullptr, RowMap{}};
    if (const int rc = launch_shrink(p, dtype, dtype, s, what)) return rc;
    p = AdapterArgs{expert_offsets, scale, R, E, N, rank, y, y_map, b, coef, out, out_map};
    return launch_expand(p, y_dtype, dtype, s, what);
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
        const size_t need = moe_adapters_workspace_bytes(R, E, K, N, rank);
        if (!workspace || workspace_bytes < need) return fail(MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", what, need, workspace_bytes);
        if (!aligned16(workspace) || !aligned16(v)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    }
    const hipStream_t s = as_stream(stream);
    const int32_t *assignments = by_assignment ? perm_src : nullptr;
    const RowMap tokens{perm_src, k, T, x_stride}, dy_map{assignments, 1, R, dy_stride}, dx_map{assignments, 1, R, dx_stride};
    float *u = (float *)workspace;
    if (R > 0 && (dx || da)) {
        const AdapterArgs p{expert_offsets, scale, R, E, N, rank, dy, dy_map, b, u, nullptr, RowMap{}};
        if (const int rc = launch_shrink(p, dy_dtype, dtype, s, what)) return rc;
    }
    if (R > 0 && dx) {
        const AdapterArgs p{expert_offsets, nullptr, R, E, K, rank, nullptr, RowMap{}, a, u, dx, dx_map};
        if (const int rc = launch_expand(p, dtype, dtype, s, what)) return rc;
    }
    if (da) {
        const AdapterArgs p{expert_offsets, nullptr, R, E, K, rank, x, tokens, nullptr, u, da, RowMap{}};
        if (const int rc = launch_outer(p, dtype, grad_dtype, s, what)) return rc;
    }
    if (db) {
        const AdapterArgs p{expert_offsets, scale, R, E, N, rank, dy, dy_map, nullptr, const_cast<float *>(v), db, RowMap{}};
        if (const int rc = launch_outer(p, dy_dtype, grad_dtype, s, what)) return rc;
    }
    return MOE_OK;
}
