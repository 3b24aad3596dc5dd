// Low-rank adapters: rows times A, and those coefficients times B beside y, in one launch.
#pragma once

#include "moe_adapters.h"

namespace moe {

// A block takes up to 16 MT rows of an adapter and a slice of N.  Phase one: its W wavefronts split K, each with all of the rows and all of the rank, operands straight from memory in
// the matrix cores' order (both lie along K); their sums meet in LDS in a fixed order.  Phase two: the coefficients, as pairs of 16-bit numbers that stand beside each other along the
// products' inner axis (so that a product of 32 holds 16 of the rank), times B, whose columns a lane puts together from four neighbouring channels of eight of its rows.
template <int XDT, int WDT, int ODT, int W, int MT, int NT>
struct AdapterShape {
    static constexpr bool kNarrow = XDT == WDT;                  // products in 16 bits; otherwise fp32 ones, 16 channels a step instead of 32
    static constexpr int KS = kNarrow ? 32 : 16, LV = KS / 4;   // channels of a step, and of a lane
    static constexpr int U = NT <= 2 ? 4 : NT == 4 ? 2 : 1;     // steps whose operands are requested together
    static constexpr int BM = 16 * MT, J = 16 * NT, kRed = J + 4, kPairs = 2 * J + 8;      // padded against bank conflicts
    static constexpr int kLds = W * BM * kRed * 4 + BM * kPairs * 2 + BM * 4;
};

template <int XDT, int WDT, int ODT, int W, int MT, int NT>
__global__ __launch_bounds__(64 * W) void adapter_kernel(AdapterArgs p)
{
    using S = AdapterShape<XDT, WDT, ODT, W, MT, NT>;
    constexpr int BM = S::BM, J = S::J, KS = S::KS, LV = S::LV, U = S::U;
    extern __shared__ __align__(16) uint8_t lds[];
    float *red = reinterpret_cast<float *>(lds);
    uint16_t *pairs = reinterpret_cast<uint16_t *>(lds + W * BM * S::kRed * 4);
    float *unit = reinterpret_cast<float *>(lds + W * BM * S::kRed * 4 + BM * S::kPairs * 2);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 15, g = lane >> 4;
    const int K = p.K, N = p.N, rank = p.rank;

    if ((int)blockIdx.x >= p.items) {                           // rows of no adapter: y's, or 0
        const int active = min(max(p.offsets[p.E], 0), p.R);
        for (int r = active + ((int)blockIdx.x - p.items) * W + wave; r < p.R; r += (gridDim.x - p.items) * W) {
            const size_t row = p.out_map.row(r);
            for (int c = lane * 8; c < N; c += 512) {
                Raw<ODT, 8> y;
                if (p.y) y.load(p.y, row * p.y_stride + c);
                else y.clear();
                y.store(p.out, row * p.out_map.stride + c);
            }
        }
        return;
    }
    int e, col, row0, rows;
    if (!find_item<16>(p.offsets, p.E, p.R, BM, p.ncol, blockIdx.x, &e, &col, &row0, &rows)) return;
    e = __builtin_amdgcn_readfirstlane(e), col = __builtin_amdgcn_readfirstlane(col);
    row0 = __builtin_amdgcn_readfirstlane(row0), rows = __builtin_amdgcn_readfirstlane(rows);
    const float scale = p.scale ? p.scale[e] : 1.0f;

    // Phase one.
    float4_t acc[MT][NT] = {};
    {
        size_t x_at[MT];
        int w_at[NT];
        const uint16_t *w = reinterpret_cast<const uint16_t *>(p.a) + (size_t)e * rank * K;
#pragma unroll
        for (int m = 0; m < MT; ++m) x_at[m] = (size_t)p.x_map.row(row0 + min(16 * m + l, rows - 1)) * p.x_map.stride + g * LV;
#pragma unroll
        for (int n = 0; n < NT; ++n) w_at[n] = min(16 * n + l, rank - 1) * K + g * LV;      // (past the rank: the last row again, left out below)
        auto steps = [&](int k0, auto whole_c) {
            constexpr bool WHOLE = decltype(whole_c)::value;
            Raw<XDT, LV> x[U][MT];
            Raw<WDT, LV> a[U][NT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = k0 + u * KS;
                const bool in = WHOLE || k + g * LV < K;        // (a lane's channels are all inside or all outside)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    if (in) x[u][m].load(p.x, x_at[m] + k);
                    else x[u][m].clear();
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (in) a[u][n].load(w, w_at[n] + k);
                    else a[u][n].clear();
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        if constexpr (S::kNarrow) {
                            acc[m][n] = product16<WDT>(u32x4_t{x[u][m].w[0], x[u][m].w[1], x[u][m].w[2], x[u][m].w[3]},
                                                       u32x4_t{a[u][n].w[0], a[u][n].w[1], a[u][n].w[2], a[u][n].w[3]}, acc[m][n]);
                        } else {
#pragma unroll
                            for (int i = 0; i < LV; ++i) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[u][m].get(i), a[u][n].get(i), acc[m][n], 0, 0, 0);
                        }
                    }
        };
        for (int k0 = wave * U * KS; k0 < K; k0 += W * U * KS) {
            if (k0 + U * KS <= K) steps(k0, std::true_type{});
            else steps(k0, std::false_type{});
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[(wave * BM + 16 * m + 4 * g + i) * S::kRed + 16 * n + l] = acc[m][n][i];
    __syncthreads();
    {
        constexpr int TPR = 64 * W / BM, Q = (J + TPR - 1) / TPR;       // threads of a row, and what each has of the rank
        static_assert(64 % TPR == 0 && TPR <= 64, "a row's threads are lanes of one wavefront");
        const int row = threadIdx.x / TPR, j0 = threadIdx.x % TPR;
        float c[Q], most = 0.0f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int j = j0 + q * TPR;
            float sum = 0.0f;
            if (j < J) {
#pragma unroll
                for (int w = 0; w < W; ++w) sum += red[(w * BM + row) * S::kRed + j];
            }
            const bool in = j < rank && row < rows;
            c[q] = in ? scale * sum : 0.0f;
            if (in && p.coef && col == 0) p.coef[(size_t)(row0 + row) * rank + j] = p.coef_scaled ? c[q] : sum;
            most = fmaxf(most, fabsf(c[q]));
        }
        float back = 1.0f;
        if constexpr (WDT == MOE_F16) {                         // fp16: a power of two per row
#pragma unroll
            for (int m = TPR / 2; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
            const int ex = split_exponent(most);
            back = exp2i(-ex);
            if (j0 == 0) unit[row] = exp2i(ex);
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int j = j0 + q * TPR;
            if (j >= J) continue;
            const Split<WDT> s(WDT == MOE_F16 ? c[q] * back : c[q]);
            uint16_t *at = pairs + row * S::kPairs + (j >> 4) * 32 + (j & 15);          // sixteen of the rank: their hi, then their lo
            at[0] = s.hi, at[16] = s.lo;
        }
    }
    if (!p.out) return;                                         // (coefficients alone)
    __syncthreads();

    // Phase two.
    u32x4_t coef[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) coef[m][n] = *reinterpret_cast<const u32x4_t *>(pairs + (16 * m + l) * S::kPairs + 32 * n + 8 * g);
    int out_row[MT][4];
    float power[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * m + 4 * g + i;
            out_row[m][i] = r < rows ? p.out_map.row(row0 + r) : -1;
            if constexpr (WDT == MOE_F16) power[m][i] = unit[r];
        }
    const uint16_t *b = reinterpret_cast<const uint16_t *>(p.b) + (size_t)e * rank * N;
    const int end = min(N, (col + 1) * p.width);
    for (int c0 = col * p.width + wave * 64; c0 < end; c0 += 64 * W) {
        const int c = c0 + 4 * l;
        const bool in = c < end;
        Raw<ODT, 4> y[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (p.y && in && out_row[m][i] >= 0) y[m][i].load(p.y, (size_t)out_row[m][i] * p.y_stride + c);
                else y[m][i].clear();
            }
        float4_t sum[MT][4] = {};                               // [..][t]: column c + t
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint2 row[8];
            u32x4_t column[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 16 * n + 8 * (g & 1) + i;
                row[i] = j < rank && in ? *reinterpret_cast<const uint2 *>(b + (j * N + c)) : make_uint2(0, 0);
            }
            transpose_8x4(row, column);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int m = 0; m < MT; ++m) sum[m][t] = product16<WDT>(coef[m][n], column[t], sum[m][t]);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!in || out_row[m][i] < 0) continue;
                float v[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) v[t] = y[m][i].get(t) + (WDT == MOE_F16 ? sum[m][t][i] * power[m][i] : sum[m][t][i]);
                y[m][i].set(v);
                y[m][i].store(p.out, (size_t)out_row[m][i] * p.out_map.stride + c);
            }
    }
}

template <int XDT, int WDT, int ODT, int W, int MT, int NT>
static int launch_adapter_shape(AdapterArgs p, int slices, hipStream_t s, const char *what)
{
    using S = AdapterShape<XDT, WDT, ODT, W, MT, NT>;
    if (!p.out) slices = 1;
    p.width = (int)round_up(((size_t)p.N + slices - 1) / slices, 64);
    p.ncol = (p.N + p.width - 1) / p.width;
    const long slots = (long)p.R / S::BM + (p.E < p.R ? p.E : p.R);
    const long items = (slots * p.ncol + kXcds - 1) / kXcds * kXcds;             // upper bound of the work items, whole rounds of XCDs
    const long copies = p.y == p.out || !p.out ? 0 : (p.R + W - 1) / W < 256 ? (p.R + W - 1) / W : 256;
    if ((items + copies) * W > 0x3ffffff) return fail(MOE_ERR_UNSUPPORTED, "%s: %ld workgroups exceed one launch", what, items);
    p.items = (int)items;
    static std::atomic<uint64_t> raised;
    const auto kernel = &adapter_kernel<XDT, WDT, ODT, W, MT, NT>;
    if (S::kLds > 64 * 1024) raise_lds_limit(reinterpret_cast<const void *>(kernel), S::kLds, raised);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(items + copies)), dim3(64 * W), S::kLds, s, p);
    return check_launch(what);
}

template <int XDT, int WDT, int ODT>
static int launch_adapter_types(const AdapterArgs &p, hipStream_t s, const char *what)
{
    auto shape = [&](auto w_c, auto mt_c, int slices) {
        constexpr int W = decltype(w_c)::value, MT = decltype(mt_c)::value;
        if (p.rank <= 16) return launch_adapter_shape<XDT, WDT, ODT, W, MT, 1>(p, slices, s, what);
        if (p.rank <= 32) return launch_adapter_shape<XDT, WDT, ODT, W, MT, 2>(p, slices, s, what);
        if (p.rank <= 64) return launch_adapter_shape<XDT, WDT, ODT, W, MT, 4>(p, slices, s, what);
        return launch_adapter_shape<XDT, WDT, ODT, W, MT, 8>(p, slices, s, what);
    };
    using std::integral_constant;
    // tiles that rows spread evenly over the adapters would make
    const long few = p.R / 16 + (p.E < p.R ? p.E : p.R);
    if (few <= 256) return shape(integral_constant<int, 16>{}, integral_constant<int, 1>{}, (int)(256 / few < 8 ? 256 / few : 8));
    return shape(integral_constant<int, 4>{}, integral_constant<int, 2>{}, 1);
}

// Rows of x and y in the adapters' own type or fp32, and, of backward passes, the other way round; other pairs of 16-bit types as well.
template <int WDT>
static int launch_adapter(const AdapterArgs &p, int x_dtype, int out_dtype, hipStream_t s, const char *what)
{
    if (x_dtype == WDT) return with_dtype(out_dtype, [&](auto o) { return launch_adapter_types<WDT, WDT, decltype(o)::value>(p, s, what); });
    return with_dtype(x_dtype, [&](auto x) {
        constexpr int X = decltype(x)::value;
        if constexpr (X == WDT) return (int)MOE_ERR_UNSUPPORTED;
        else return launch_adapter_types<X, WDT, WDT>(p, s, what);              // (backward: dx has the adapters' type)
    });
}

}  // namespace moe
