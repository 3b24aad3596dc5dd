// moe_combine_backward, moe_permute_backward: the gradient of sorting tokens by expert and back.
//
//   out[t] = sum_j s[t,j] y[inv[t k + j]]:  dy[inv[a]] = s[a] dout[a / k],  ds[a] = <dout[a / k], y[inv[a]]>
//   x_perm[r] = x[perm_src[r] / k]:         dx[t] = sum_j dx_perm[inv[t k + j]]
//
// Both go by token: a token's k rows are written by nobody else, so nothing is added into memory and the sums have one order.  One pass over the data each, bound by memory (16384 tokens of
// 4096, two rows each, fp16: 671 MB in 144 us = 4.7 TB/s, 403 MB in 88 us = 4.6 TB/s) or, for small batches, by a launch (512 tokens of 256: 3.6 and 3.1 us).
#include "moe_rows.h"

namespace moe {

struct ExchangeArgs {
    const void *dout;               // [T, d]
    const void *y;                  // [R, d]: y_perm, or dx_perm
    const int32_t *inv;             // [T k]
    const float *scale;             // [T k]
    const int32_t *active_rows;     // [1] or null
    int T, k, d, R;
    void *dy;                       // [R, d] or null
    float *dscale;                  // [T k] or null
    void *dx;                       // [T, d]
};

// A wavefront per token; ds is summed over its lanes.  K: rows of a token, 0 for any number, one after the other.  With K known a step's loads of all of its rows are requested together.
template <int ODT, int YDT, int K>
__global__ __launch_bounds__(256) void combine_backward_kernel(ExchangeArgs p)
{
    constexpr int V = ODT == MOE_F32 || YDT == MOE_F32 ? 4 : 8, N = K ? K : 1;
    const int lane = threadIdx.x & 63, steps = p.d / V;
    const int active = min(p.active_rows ? *p.active_rows : p.R, p.R);
    for (uint32_t t = blockIdx.x * 4 + (threadIdx.x >> 6); t < (uint32_t)p.T; t += gridDim.x * 4) {       // (unsigned: T and a stride of up to 2^22 stay below 2^32)
        for (int j0 = 0; j0 < (K ? 1 : p.k); ++j0) {
            const size_t a = (size_t)t * (K ? K : p.k) + j0;
            int r[N];
            float s[N], sum[N] = {};
            bool live[N];
#pragma unroll
            for (int j = 0; j < N; ++j) r[j] = p.inv[a + j], s[j] = p.scale[a + j];
#pragma unroll
            for (int j = 0; j < N; ++j) live[j] = r[j] >= 0 && r[j] < active;
#pragma unroll 2
            for (int c = lane; c < steps; c += 64) {
                Raw<ODT, V> o;
                Raw<YDT, V> y[N];
                o.load(p.dout, (size_t)t * p.d + c * V);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (p.dscale && live[j]) y[j].load(p.y, (size_t)r[j] * p.d + c * V);
                    else y[j].clear();
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float v[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[j] = live[j] ? fmaf(o.get(i), y[j].get(i), sum[j]) : 0.0f, v[i] = live[j] ? s[j] * o.get(i) : 0.0f;
                    if (p.dy && r[j] >= 0 && r[j] < p.R) y[j].set(v), y[j].store(p.dy, (size_t)r[j] * p.d + c * V);
                }
            }
            if (!p.dscale) continue;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                sum[j] = wave_sum(sum[j]);
                if (lane == 0) p.dscale[a + j] = sum[j];
            }
        }
    }
}

template <int YDT, int ODT>
__global__ __launch_bounds__(256) void permute_backward_kernel(ExchangeArgs p)
{
    constexpr int V = YDT == MOE_F32 ? 4 : 8;
    const size_t steps = p.d / V, total = p.T * steps;
    const int active = min(p.active_rows ? *p.active_rows : p.R, p.R);
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const size_t t = i / steps, c = i - t * steps;
        float sum[V] = {};
        for (int j = 0; j < p.k; ++j) {
            const int r = p.inv[t * p.k + j];
            if (r < 0 || r >= active) continue;
            Raw<YDT, V> y;
            y.load(p.y, (size_t)r * p.d + c * V);
#pragma unroll
            for (int q = 0; q < V; ++q) sum[q] += y.get(q);
        }
        Raw<ODT, V> out;
        out.set(sum);
        out.store(p.dx, i * V);
    }
}

static int check_exchange(const char *what, int T, int k, int d, int R, int in_dtype, int out_dtype)
{
    if (T < 0 || R < 0 || k <= 0 || d <= 0 || d % 8) return fail(MOE_ERR_INVALID_ARG, "%s: need T, R >= 0, k > 0, d > 0, d %% 8 == 0", what);
    if ((long long)T * k > 0x7fffffffLL) return fail(MOE_ERR_INVALID_ARG, "%s: T*k overflows int32", what);
    if (!known_dtype(in_dtype) || !known_dtype(out_dtype)) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    return MOE_OK;
}

}  // namespace moe

extern "C" int moe_combine_backward(const void *dout, int out_dtype, const void *y_perm, int y_dtype, const int32_t *inv_perm, const float *expert_scale,
                                    const int32_t *active_rows, int T, int k, int d, int R, void *dy_perm, float *dscale, void *stream)
{
    using namespace moe;
    const char *what = "moe_combine_backward";
    if (const int rc = check_exchange(what, T, k, d, R, out_dtype, y_dtype)) return rc;
    if (T == 0) return MOE_OK;                                      // empty buffers may be NULL
    if (!dout || !inv_perm || !expert_scale || (!dscale && !dy_perm) || (R > 0 && dscale && !y_perm)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(dout) || !aligned16(y_perm) || !aligned16(dy_perm)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const ExchangeArgs p{dout, y_perm, inv_perm, expert_scale, active_rows, T, k, d, R, dy_perm, dscale, nullptr};
    const int blocks = (int)(((long)T + 3) / 4 < 0x100000 ? ((long)T + 3) / 4 : 0x100000);
    return with_dtype(out_dtype, [&](auto o) {
        return with_dtype(y_dtype, [&](auto y) {
            constexpr int O = decltype(o)::value, Y = decltype(y)::value;
            const auto kernel = k == 1 ? &combine_backward_kernel<O, Y, 1> : k == 2 ? &combine_backward_kernel<O, Y, 2> : &combine_backward_kernel<O, Y, 0>;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, as_stream(stream), p);
            return check_launch(what);
        });
    });
}

extern "C" int moe_permute_backward(const void *dx_perm, int perm_dtype, const int32_t *inv_perm, const int32_t *active_rows, int T, int k, int d, int R,
                                    void *dx, int dx_dtype, void *stream)
{
    using namespace moe;
    const char *what = "moe_permute_backward";
    if (const int rc = check_exchange(what, T, k, d, R, perm_dtype, dx_dtype)) return rc;
    if (T == 0) return MOE_OK;
    if (!inv_perm || !dx || (R > 0 && !dx_perm)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(dx_perm) || !aligned16(dx)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const ExchangeArgs p{nullptr, dx_perm, inv_perm, nullptr, active_rows, T, k, d, R, nullptr, nullptr, dx};
    const size_t blocks = ((size_t)T * (d / 4) + 255) / 256;
    return with_dtype(perm_dtype, [&](auto y) {
        return with_dtype(dx_dtype, [&](auto o) {
            hipLaunchKernelGGL((permute_backward_kernel<decltype(y)::value, decltype(o)::value>), dim3((unsigned)(blocks < 0x400000 ? blocks : 0x400000)), dim3(256), 0,
                               as_stream(stream), p);
            return check_launch(what);
        });
    });
}
