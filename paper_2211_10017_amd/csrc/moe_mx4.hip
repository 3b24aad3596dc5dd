// moe_grouped_gemm_mx4, moe_grouped_ffn_mx4: checks of their arguments, the workspace and the chain of launches.
#include "moe_mx4_common.h"

namespace moe {

static int check_product(const char *what, int R, int E, int a_rows, int K, int N, const int32_t *perm_src, int k)
{
    if (R < 0 || E < 0 || a_rows < 0 || K <= 0 || N <= 0 || K % 64 || N % 32)
        return fail(MOE_ERR_INVALID_ARG, "%s: need R, E and rows >= 0, K %% 64 == 0, N %% 32 == 0 (R=%d E=%d rows=%d K=%d N=%d)", what, R, E, a_rows, K, N);
    if (perm_src ? k < 1 : a_rows < R) return fail(MOE_ERR_INVALID_ARG, "%s: without perm_src there are as many rows as R, with it k >= 1", what);
    if (K > 1 << 24 || N > 1 << 24) return fail(MOE_ERR_UNSUPPORTED, "%s: K = %d or N = %d above 2^24", what, K, N);      // (what a lane's 32-bit offsets reach)
    if (a_rows > 0x3fffffff) return fail(MOE_ERR_UNSUPPORTED, "%s: %d rows are 2^30 or more", what, a_rows);
    if (E > 4096) return fail(MOE_ERR_UNSUPPORTED, "%s: E = %d above 4096", what, E);
    return MOE_OK;
}

// Rows that there can be: R, or less where the caller bounds every expert's.
static int most_rows(int R, int E, int max_rows_per_expert)
{
    return max_rows_per_expert && (long)E * max_rows_per_expert < R ? E * max_rows_per_expert : R;
}

}  // namespace moe

extern "C" int moe_grouped_gemm_mx4(const void *a_codes, const void *a_scales, int a_rows, const int32_t *perm_src, int k, const int32_t *expert_offsets,
                                    int R, int E, int max_rows_per_expert, int K, int N, const void *w_codes, const void *w_scales, const void *bias,
                                    int activation, void *y, int y_dtype, void *stream)
{
    using namespace moe;
    const char *what = "moe_grouped_gemm_mx4";
    if (int rc = check_product(what, R, E, a_rows, K, N, perm_src, k)) return rc;
    if (y_dtype < 0 || y_dtype > 2) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (activation < MOE_ACT_NONE || activation > MOE_ACT_GELU) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown activation %d", what, activation);
    if (max_rows_per_expert < 0) return fail(MOE_ERR_INVALID_ARG, "%s: max_rows_per_expert < 0", what);
    if (R == 0 || E == 0 || a_rows == 0) return MOE_OK;
    if (!a_codes || !a_scales || !expert_offsets || !w_codes || !w_scales || !y) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(w_codes) || !aligned16(w_scales) || !aligned16(y) || !aligned16(bias))
        return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    MxArgs p{};
    p.a = (const uint8_t *)a_codes, p.as = (const uint8_t *)a_scales, p.a_rows = a_rows, p.a_src = perm_src, p.a_div = k;
    p.offsets = expert_offsets, p.w = (const uint8_t *)w_codes, p.ws = (const uint8_t *)w_scales, p.bias = (const __half *)bias;
    p.out = y, p.E = E, p.R = R, p.most = most_rows(R, E, max_rows_per_expert), p.K = K, p.N = N, p.out_dtype = y_dtype, p.act = activation;
    return launch_mx4_gemm(p, as_stream(stream));
}

extern "C" size_t moe_grouped_ffn_mx4_workspace_bytes(int T, int R, int d, int F)
{
    using namespace moe;
    if (T < 0 || R < 0 || d <= 0 || F <= 0) return 0;
    return round_up(mx_code_bytes(T, d), 256) + round_up(mx_scale_bytes(T, d), 256) + round_up(mx_code_bytes(R, F), 256) + round_up(mx_scale_bytes(R, F), 256);
}

extern "C" int moe_grouped_ffn_mx4(const void *x, int act_dtype, int T, const int32_t *perm_src, int k, const int32_t *expert_offsets, int R, int E,
                                   int max_rows_per_expert, int d, int F, int activation, const void *w1_codes, const void *w1_scales, const void *b1,
                                   const void *w2_codes, const void *w2_scales, const void *b2, void *y_perm, int y_dtype, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    using namespace moe;
    const char *what = "moe_grouped_ffn_mx4";
    if (int rc = check_product(what, R, E, T, d, F, perm_src, k)) return rc;
    if (F % 64) return fail(MOE_ERR_INVALID_ARG, "%s: F must be a multiple of 64", what);
    if (R > 0x3fffffff) return fail(MOE_ERR_UNSUPPORTED, "%s: %d rows are 2^30 or more", what, R);       // (fc2's rows are h's)
    if (act_dtype < 0 || act_dtype > 2 || y_dtype < 0 || y_dtype > 2) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (activation < MOE_ACT_RELU || activation > MOE_ACT_GELU) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown activation %d", what, activation);
    if (max_rows_per_expert < 0) return fail(MOE_ERR_INVALID_ARG, "%s: max_rows_per_expert < 0", what);
    if (R == 0 || E == 0 || T == 0) return MOE_OK;
    if (!x || !expert_offsets || !w1_codes || !w1_scales || !w2_codes || !w2_scales || !y_perm) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    for (const void *b : {x, w1_codes, w1_scales, b1, w2_codes, w2_scales, b2, (const void *)y_perm, (const void *)workspace})
        if (!aligned16(b)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const size_t need = moe_grouped_ffn_mx4_workspace_bytes(T, R, d, F);
    if (!workspace || workspace_bytes < need) return fail(MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", what, workspace ? workspace_bytes : (size_t)0, need);
    hipStream_t s = as_stream(stream);
    uint8_t *xq = (uint8_t *)workspace, *xs = xq + round_up(mx_code_bytes(T, d), 256);
    uint8_t *hq = xs + round_up(mx_scale_bytes(T, d), 256), *hs = hq + round_up(mx_code_bytes(R, F), 256);
    MxArgs p{};
    p.most = most_rows(R, E, max_rows_per_expert);
    if (mx4_fuses_rows(p.most, E, F, act_dtype)) p.x = x, p.x_dtype = act_dtype;
    else if (int rc = launch_mx4_quantize_rows(x, act_dtype, T, d, d, xq, xs, s)) return rc;
    p.a = xq, p.as = xs, p.a_rows = T, p.a_src = perm_src, p.a_div = k, p.offsets = expert_offsets;
    p.w = (const uint8_t *)w1_codes, p.ws = (const uint8_t *)w1_scales, p.bias = (const __half *)b1;
    p.out = hq, p.out_scales = hs, p.E = E, p.R = R, p.K = d, p.N = F, p.act = activation;
    if (int rc = launch_mx4_gemm(p, s)) return rc;
    p.x = nullptr, p.a = hq, p.as = hs, p.a_rows = R, p.a_src = nullptr, p.w = (const uint8_t *)w2_codes, p.ws = (const uint8_t *)w2_scales, p.bias = (const __half *)b2;
    p.out = y_perm, p.out_scales = nullptr, p.out_dtype = y_dtype, p.K = F, p.N = d, p.act = MOE_ACT_NONE;
    return launch_mx4_gemm(p, s);
}
