// Low-rank adapters: rows times A, and those coefficients times B beside y, in one launch.
#pragma once

#include "moe_adapters.h"

namespace moe {

// ---- phase one: rows times A ---------------------------------------------------------------------------------------------------------------------

// acc[m][n] += rows 16 m.. of the item times the rows first + 16 n.. of A[e], over this wavefront's share of K: of every 4 W steps the four that are its own.  Operands come straight from memory
// in the matrix cores' order (both lie along K) and stay D steps ahead of their products: a step's registers are requested anew as soon as it has been multiplied.
template <int XDT, int WDT, int D, int W, int MT, int NT>
__device__ inline void multiply_rows(const AdapterArgs &p, int e, int first, int row0, int rows, int wave, float4_t (&acc)[MT][NT])
{
    constexpr bool kNarrow = XDT == WDT;                        // products in 16 bits; otherwise fp32 ones, 16 channels a step instead of 32
    constexpr int KS = kNarrow ? 32 : 16, LV = KS / 4;          // channels of a step, and of a lane
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, K = p.K, rank = p.rank;
    int x_row[MT], w_at[NT];
    size_t x_at[MT];
    const uint16_t *w = reinterpret_cast<const uint16_t *>(p.a) + (size_t)e * rank * K;
#pragma unroll
    for (int m = 0; m < MT; ++m) x_row[m] = row0 + min(16 * m + l, rows - 1);
    p.x_map.find(x_row);
#pragma unroll
    for (int m = 0; m < MT; ++m) x_at[m] = (size_t)x_row[m] * p.x_map.stride + g * LV;
#pragma unroll
    for (int n = 0; n < NT; ++n) w_at[n] = min(first + 16 * n + l, rank - 1) * K + g * LV;      // (past the rank: the last row again, left out by the caller)
    Raw<XDT, LV> x[D][MT];
    Raw<WDT, LV> a[D][NT];
    const int steps = K / KS, own = steps / (4 * W) * 4 + min(max(steps % (4 * W) - 4 * wave, 0), 4);
    auto request = [&](auto u_c, int i) {
        constexpr int B = decltype(u_c)::value;
        const int k = ((i >> 2) * 4 * W + wave * 4 + (i & 3)) * KS;
#pragma unroll
        for (int n = 0; n < NT; ++n) a[B][n].load(w, w_at[n] + k);
#pragma unroll
        for (int m = 0; m < MT; ++m) x[B][m].load(p.x, x_at[m] + k);
        requested();
    };
    auto use = [&](auto u_c) {
        constexpr int B = decltype(u_c)::value;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (kNarrow) {
                    acc[m][n] = product16<WDT>(u32x4_t{x[B][m].w[0], x[B][m].w[1], x[B][m].w[2], x[B][m].w[3]}, u32x4_t{a[B][n].w[0], a[B][n].w[1], a[B][n].w[2], a[B][n].w[3]}, acc[m][n]);
                } else {
#pragma unroll
                    for (int i = 0; i < LV; ++i) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[B][m].get(i), a[B][n].get(i), acc[m][n], 0, 0, 0);
                }
            }
        requested();
    };
    if (own > 0) {
        unrolled<D>([&](auto u) { request(u, min((int)decltype(u)::value, own - 1)); });
        int i = 0;
        for (; i + D < own; i += D)
            unrolled<D>([&](auto u) { use(u), request(u, min(i + D + (int)decltype(u)::value, own - 1)); });
        unrolled<D>([&](auto u) {
            if (i + (int)decltype(u)::value < own) use(u);
        });
    }
    if (K % KS && (steps >> 2) % W == wave) {                   // channels behind the last whole step
        const int k = steps * KS;
        const bool in = k + g * LV < K;                         // (a lane's channels are all inside or all outside)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (in) a[0][n].load(w, w_at[n] + k);
            else a[0][n].clear();
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (in) x[0][m].load(p.x, x_at[m] + k);
            else x[0][m].clear();
        }
        use(std::integral_constant<int, 0>{});
    }
}

// ---- what both kernels below hold in LDS ---------------------------------------------------------------------------------------------------------

template <int WDT, int ODT, int W, int MT, int NT>
struct AdapterShape {
    static constexpr int BM = 16 * MT, J = 16 * NT;             // rows, and the rank in whole products
    static constexpr int D = (W == 16 ? 40 : 96) / (4 * (MT + NT)) < 2 ? 2 : (W == 16 ? 40 : 96) / (4 * (MT + NT)) > 6 ? 6 : (W == 16 ? 40 : 96) / (4 * (MT + NT));
    static constexpr int kParts = W == 8 && NT >= 4 ? W / 2 : W, kRed = J + 4;              // wavefronts' sums at a time; rows padded against bank conflicts
    static constexpr int CL = ODT != MOE_F32 && W == 8 && NT <= 2 ? 8 : 4;                   // channels of a lane in phase two
    static constexpr int KI = NT == 1 ? 16 : 32, NC = J / KI, JL = KI / 4;                  // phase two: inner size of a product, products over the rank, rank of a lane in one
    static constexpr int TERMS = WDT == MOE_BF16 && ODT == MOE_F32 ? 3 : 2, kTermRow = TERMS * J + 8;
    static constexpr int kTerms = kParts * BM * kRed * 4, kUnit = kTerms + BM * kTermRow * 2, kPlace = kUnit + BM * 4, kLds = kPlace + BM * 16;
};

// A row's coefficients, TPR lanes' worth of them, as 16-bit terms in LDS.
template <class S, int WDT, int TPR, int Q>
__device__ inline void store_terms(uint8_t *lds, const float (&c)[Q], float most, int row, int j0)
{
    float *unit = reinterpret_cast<float *>(lds + S::kUnit);
    uint16_t *terms = reinterpret_cast<uint16_t *>(lds + S::kTerms);
    constexpr int J = S::J;
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
        uint16_t *to = terms + row * S::kTermRow + j;
        to[0] = s.hi, to[J] = s.lo;
        if constexpr (S::TERMS == 3) to[2 * J] = s.rest;
    }
}

// The wavefronts' sums become coefficients: added in a fixed order, written to memory if they are wanted there, and left in LDS as 16-bit terms.
// `first`: of the rank, where coefficients alone are wanted, a part of it.
template <class S, int WDT, int W, int MT, int NT>
__device__ inline void make_terms(const AdapterArgs &p, uint8_t *lds, float4_t (&acc)[MT][NT], int e, int first, int row0, int rows, int wave, bool keep)
{
    constexpr int BM = S::BM, J = S::J, P = S::kParts, TPR = 64 * W / BM >= 64 ? 64 : 64 * W / BM >= 32 ? 32 : 64 * W / BM >= 16 ? 16 : 8, Q = (J + TPR - 1) / TPR;
    static_assert(64 * W >= BM * TPR || TPR == 8, "a row's threads are lanes of one wavefront");
    float *red = reinterpret_cast<float *>(lds);
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, rank = p.rank;
    auto at = [&](int part, int m, int n, int i) -> float & { return red[(part * BM + 16 * m + 4 * g + i) * S::kRed + 16 * n + l]; };
    auto put = [&](int part) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) at(part, m, n, i) = acc[m][n][i];
    };
    if constexpr (P == W) put(wave);
    else {                                                      // (the second half's first where all would be too much)
        if (wave >= P) put(wave - P);
        __syncthreads();
        if (wave < P) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][n][i] += at(wave, m, n, i);
            put(wave);                                          // (each place is read and written by the same lane)
        }
    }
    __syncthreads();
    const float scale = p.scale ? p.scale[e] : 1.0f;
    const int j0 = threadIdx.x % TPR;
    for (int row = threadIdx.x / TPR; row < BM; row += 64 * W / TPR) {
        float c[Q], most = 0.0f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int j = j0 + q * TPR;
            float sum = 0.0f;
            if (j < J) {
#pragma unroll
                for (int w = 0; w < P; ++w) sum += red[(w * BM + row) * S::kRed + j];
            }
            const bool in = j < J && first + j < rank && row < rows;
            c[q] = in ? scale * sum : 0.0f;
            if (in && keep) p.coef[(size_t)(row0 + row) * rank + first + j] = p.coef_scaled ? c[q] : sum;
            most = fmaxf(most, fabsf(c[q]));
        }
        if (!p.out) continue;                                   // (coefficients alone)
        store_terms<S, WDT, TPR, Q>(lds, c, most, row, j0);
    }
}

// Coefficients that are in memory, as terms in LDS.
template <class S, int WDT, int W>
__device__ inline void load_terms(const AdapterArgs &p, uint8_t *lds, int e, int row0, int rows)
{
    constexpr int TPR = 64, Q = (S::J + TPR - 1) / TPR;
    const float scale = p.scale && !p.coef_scaled ? p.scale[e] : 1.0f;
    const int j0 = threadIdx.x % TPR;
    for (int row = threadIdx.x / TPR; row < S::BM; row += 64 * W / TPR) {
        float c[Q], most = 0.0f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int j = j0 + q * TPR;
            c[q] = j < p.rank && row < rows ? scale * p.coef[(size_t)(row0 + row) * p.rank + j] : 0.0f;
            most = fmaxf(most, fabsf(c[q]));
        }
        store_terms<S, WDT, TPR, Q>(lds, c, most, row, j0);
    }
}

// Phase two: coefficients times B, 16 CL channels at a time, every W-th of them from `first` to `end`.  A lane puts B's columns together from CL neighbouring channels of its rows, once for
// all of the item's rows.  The next channels' operands are requested as soon as this one's registers are free.
template <class S, int WDT, int ODT, bool Y, int W, int MT>
__device__ inline void expand_rows(const AdapterArgs &p, const uint8_t *lds, int e, int rows, int wave, int first, int end)
{
    constexpr int J = S::J, KI = S::KI, NC = S::NC, JL = S::JL, CL = S::CL;
    typedef uint32_t operand_t __attribute__((ext_vector_type(JL / 2)));
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, N = p.N, rank = p.rank;
    const uint16_t *terms = reinterpret_cast<const uint16_t *>(lds + S::kTerms), *b = reinterpret_cast<const uint16_t *>(p.b) + (size_t)e * rank * N;
    const float *unit = reinterpret_cast<const float *>(lds + S::kUnit);
    const size_t *place = reinterpret_cast<const size_t *>(lds + S::kPlace);                // of the rows in y and in out
    const int groups = (end - first + 16 * CL - 1) / (16 * CL);
    if (wave >= groups) return;
    Raw<ODT, CL> y[MT][4];
    Raw<WDT, CL> raw[NC][JL];
    auto channel = [&](int group) { return min(first + (group * 16 + l) * CL, end - CL); };          // (past the end: the last ones again, which are not stored)
    auto request_b = [&](int group) {
        const int c = channel(group);
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int i = 0; i < JL; ++i) raw[n][i].load(b, (size_t)(uint32_t)(min(KI * n + JL * g + i, rank - 1) * N + c));
        requested();
    };
    auto request_y = [&](auto m_c, int group) {
        constexpr int M = decltype(m_c)::value;
        if constexpr (Y) {
            const int c = channel(group);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[M][i].load(p.y, place[2 * (16 * M + 4 * g + i)] + c);
            requested();
        }
    };
    auto step = [&](int group, auto more_c) {
        constexpr bool MORE = decltype(more_c)::value;
        const int c = first + (group * 16 + l) * CL;
        operand_t column[NC][CL];
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int q = 0; q < CL / 4; ++q) {
                uint2 four[JL];
                operand_t out[4];
#pragma unroll
                for (int i = 0; i < JL; ++i) {
                    const bool in = KI * n + JL * g + i < rank;                 // (past the rank coefficients are 0, and 0 times an infinity is none)
                    four[i] = make_uint2(in ? raw[n][i].w[2 * q] : 0, in ? raw[n][i].w[2 * q + 1] : 0);
                }
                transpose_columns(four, out);
#pragma unroll
                for (int t = 0; t < 4; ++t) column[n][4 * q + t] = out[t];
            }
        if constexpr (MORE) request_b(group + W);
        unrolled<MT>([&](auto m_c) {
            constexpr int M = decltype(m_c)::value;
            float4_t sum[CL] = {};                              // [t]: column c + t
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int i = 0; i < S::TERMS; ++i) {
                    const operand_t coef = *reinterpret_cast<const operand_t *>(terms + (16 * M + l) * S::kTermRow + i * J + KI * n + JL * g);
#pragma unroll
                    for (int t = 0; t < CL; ++t) sum[t] = product16<WDT>(coef, column[n][t], sum[t]);
                }
            Raw<ODT, CL> out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[CL];
#pragma unroll
                for (int t = 0; t < CL; ++t) {
                    v[t] = WDT == MOE_F16 ? sum[t][i] * unit[16 * M + 4 * g + i] : sum[t][i];
                    if constexpr (Y) v[t] += y[M][i].get(t);
                }
                out[i].set(v);
            }
            if constexpr (MORE) request_y(m_c, group + W);
            if (16 * M + 16 <= rows && first + group * 16 * CL + 16 * CL <= end) {
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i].store(p.out, place[2 * (16 * M + 4 * g + i) + 1] + c);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * M + 4 * g + i < rows && c < end) out[i].store(p.out, place[2 * (16 * M + 4 * g + i) + 1] + c);
            }
            requested();
        });
    };
    int t = wave;
    request_b(t);
    unrolled<MT>([&](auto m) { request_y(m, t); });
    for (; t + W < groups; t += W) step(t, std::true_type{});
    step(t, std::false_type{});
}

// Where the item's rows are in y and in out, for phase two.
template <class S>
__device__ inline void find_places(const AdapterArgs &p, uint8_t *lds, int row0, int rows)
{
    size_t *place = reinterpret_cast<size_t *>(lds + S::kPlace);
    for (int i = threadIdx.x; i < S::BM; i += blockDim.x) {
        int r[1] = {row0 + min(i, rows - 1)};
        p.out_map.find(r);
        place[2 * i] = (size_t)r[0] * p.y_stride, place[2 * i + 1] = (size_t)r[0] * p.out_map.stride;
    }
}

// Rows of no adapter: y's, or 0.
template <int ODT, bool Y>
__device__ inline void copy_rows(const AdapterArgs &p, int block, int waves)
{
    const int lane = threadIdx.x & 63, active = min(max(p.offsets[p.E], 0), p.R);
    for (int r = active + block * waves + (threadIdx.x >> 6); r < p.R; r += (gridDim.x - p.items) * waves) {
        int at[1] = {r};
        p.out_map.find(at);
        const size_t row = at[0];
        for (int c = lane * 8; c < p.N; c += 512) {
            Raw<ODT, 8> y;
            if (Y) y.load(p.y, row * p.y_stride + c);
            else y.clear();
            y.store(p.out, row * p.out_map.stride + c);
        }
    }
}

// ---- one launch: a block takes rows of an adapter and a slice of N, its W wavefronts split K and the slice ---------------------------------------------
//
// All blocks run at once, one per compute unit where there are as many, and share the memory's rate, so the one with the most to read is waited for: an adapter's rows are cut into as many
// parts of `share` rows as come nearest, evenly, rather than into full tiles and a rest.  Neighbouring parts lie on one XCD (as find_item deals them), whose cache then holds their adapter.
// (16384 rows of 4096 x 4096, 32 adapters of rank 32, bf16 in place: 108 us = 3.7 TB/s of x and y; tiles of 16 rows of one adapter each 141: they read A and B, through the caches, twice as often as x and y.
// Wavefronts spend 55 % of their time waiting to issue loads and stores and 23 % waiting for them: the blocks' phases, all reading and then all writing, are what is left.)

// The block's adapter, slice and rows.  Every wavefront computes the same.
__device__ inline bool find_share(const AdapterArgs &p, int most, int *e, int *col, int *row0, int *rows)
{
    const int lane = threadIdx.x & 63;
    int lo, hi, parts, incl;                                    // this lane's adapter of a chunk of 64: its rows, its parts, and the chunk's parts up to its own
    auto load = [&](int e0) {
        lo = hi = 0;
        if (e0 + lane < p.E) expert_range(p.offsets, e0 + lane, p.R, &lo, &hi);
        const int n = hi - lo;
        parts = n ? max(max((n + p.share / 2) / p.share, (n + most - 1) / most), 1) : 0;
        incl = wave_inclusive_sum(parts);
    };
    load(0);
    const int lo0 = lo, hi0 = hi, parts0 = parts, incl0 = incl;             // (with up to 64 adapters the offsets are read once)
    int total = __shfl(incl, 63);
    for (int e0 = 64; e0 < p.E; e0 += 64) load(e0), total += __shfl(incl, 63);
    const int chunk = (total * p.ncol + kXcds - 1) / kXcds, within = blockIdx.x / kXcds, item = blockIdx.x % kXcds * chunk + within;
    if (within >= chunk || item >= total * p.ncol) return false;
    const int part = item / p.ncol;
    int base = 0;
    for (int e0 = 0; e0 < p.E; e0 += 64) {
        if (p.E > 64) load(e0);
        else lo = lo0, hi = hi0, parts = parts0, incl = incl0;
        const uint64_t hit = __ballot(base + incl > part);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            const int count = __shfl(parts, src), i = part - base - __shfl(incl - parts, src), size = __shfl(hi - lo, src), first = __shfl(lo, src);
            const int per = size / count, extra = size % count;
            *e = __builtin_amdgcn_readfirstlane(e0 + src), *col = __builtin_amdgcn_readfirstlane(item % p.ncol);
            *row0 = __builtin_amdgcn_readfirstlane(first + i * per + min(i, extra));
            *rows = __builtin_amdgcn_readfirstlane(per + (i < extra ? 1 : 0));
            return true;
        }
        base += __shfl(incl, 63);
    }
    return false;
}

template <int XDT, int WDT, int ODT, bool Y, int W, int MT, int NT>
__global__ __launch_bounds__(64 * W, W == 16 ? 4 : 2) void adapter_kernel(AdapterArgs p)
{
    using S = AdapterShape<WDT, ODT, W, MT, NT>;
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x >= p.items) return copy_rows<ODT, Y>(p, blockIdx.x - p.items, W);
    int e, col, row0, rows;
    if (!find_share(p, S::BM, &e, &col, &row0, &rows)) return;
    find_places<S>(p, lds, row0, rows);
    float4_t acc[MT][NT] = {};
    const int part = p.out ? 0 : col * S::J;                    // (coefficients alone: of a part of the rank, if there is a block for each)
    multiply_rows<XDT, WDT, S::D, W, MT, NT>(p, e, part, row0, rows, wave, acc);
    make_terms<S, WDT, W, MT, NT>(p, lds, acc, e, part, row0, rows, wave, p.coef && (!p.out || col == 0));
    if (!p.out) return;
    __syncthreads();
    expand_rows<S, WDT, ODT, Y, W, MT>(p, lds, e, rows, wave, col * p.width, min(p.N, (col + 1) * p.width));
}

// Phase two alone, of coefficients that are in memory.
template <int WDT, int ODT, bool Y, int NT>
__global__ __launch_bounds__(512, 2) void adapter_expand_kernel(AdapterArgs p)
{
    constexpr int W = 8;
    using S = AdapterShape<WDT, ODT, W, 1, NT>;
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x >= p.items) return copy_rows<ODT, Y>(p, blockIdx.x - p.items, W);
    int e, col, row0, rows;
    if (!find_share(p, S::BM, &e, &col, &row0, &rows)) return;
    find_places<S>(p, lds, row0, rows);
    load_terms<S, WDT, W>(p, lds, e, row0, rows);
    __syncthreads();
    expand_rows<S, WDT, ODT, Y, W, 1>(p, lds, e, rows, wave, col * p.width, min(p.N, (col + 1) * p.width));
}

// ---- launches --------------------------------------------------------------------------------------------------------------------------------------

template <class Kernel>
static int launch_items(Kernel kernel, std::atomic<uint64_t> &raised, AdapterArgs p, int share, int W, int lds, hipStream_t s, const char *what)
{
    p.share = share;
    const long parts = (long)p.R / share + (p.E < p.R ? p.E : p.R);             // an upper bound: of n rows at most n / share + 1
    const long items = (parts * p.ncol + kXcds - 1) / kXcds * kXcds;
    const int need = p.y == p.out || !p.out ? 0 : (p.R + W - 1) / W, copies = need < 256 ? need : 256;          // blocks for rows of no adapter
    if ((items + copies) * W > 0x3ffffff) return fail(MOE_ERR_UNSUPPORTED, "%s: %ld workgroups exceed one launch", what, items);
    p.items = (int)items;
    if (lds > 64 * 1024) raise_lds_limit(reinterpret_cast<const void *>(kernel), lds, raised);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(items + copies)), dim3(64 * W), lds, s, p);
    return check_launch(what);
}

static void cut_channels(AdapterArgs &p, int slices)
{
    p.width = (int)round_up(((size_t)p.N + slices - 1) / slices, 64);
    p.ncol = (p.N + p.width - 1) / p.width;
}

template <int XDT, int WDT, int ODT, bool Y, int W, int MT, int NT>
static int launch_shape(AdapterArgs p, int share, int slices, hipStream_t s, const char *what)
{
    static std::atomic<uint64_t> raised;
    if (p.out) cut_channels(p, slices);
    else p.ncol = (p.rank + 16 * NT - 1) / (16 * NT);
    return launch_items(&adapter_kernel<XDT, WDT, ODT, Y, W, MT, NT>, raised, p, share, W, AdapterShape<WDT, ODT, W, MT, NT>::kLds, s, what);
}

template <int WDT, int ODT, bool Y, int NT>
static int launch_expand(AdapterArgs p, int share, int slices, hipStream_t s, const char *what)
{
    static std::atomic<uint64_t> raised;
    cut_channels(p, slices);
    return launch_items(&adapter_expand_kernel<WDT, ODT, Y, NT>, raised, p, share, 8, AdapterShape<WDT, ODT, 8, 1, NT>::kLds, s, what);
}

// One block per compute unit, of the fewest rows' registers that hold its share (32 adapters of 4096 x 4096, rank 16 / 32, bf16, in blocks of up to 16, 32, 48 and 80 rows: 3000 rows, shares of 12,
// 22 / 27, 27 / 33, 34 / 38, 47 / 54 us; 3968, 16, 34 / 46, 28 / 34, 35 / 39, 48 / 55; 7000, 28, 54, 44, 47, 58; 8192, 33, 69, 60, 54, 62; 11000, 44, 81 / 103, 72 / 87, 66 / 71, 72 / 80.
// Rank 64 in blocks of up to 16, 32, 48 and 64 rows: 3968, 74, 52, 60, 68; 7000, 63 of 32, 71, 77; 8192, 110, 76, 82.  Rank 128, 16, 32 and 48: 3968, 133, 82, 97; 7000, 93 of 32, 105.)
template <int XDT, int WDT, int ODT, bool Y, int NT>
static int launch_rank(const AdapterArgs &p, hipStream_t s, const char *what)
{
    constexpr int kUnits = 248, kMost = NT <= 2 ? 80 : NT == 4 ? 64 : 48;       // a few fewer than compute units, as parts are rounded one way or the other; rows that a block can hold
    const long even = ((long)p.R + kUnits - 1) / kUnits;
    if (!p.coef || even <= 13) {
        // Few rows: parts of an adapter's rows and slices of N such that what a block moves (its rows of x, A, and its slice of y, out and B), times the rounds of blocks, is least.  What a
        // block takes to begin and to join its sums is as long as 96 KB.
        constexpr int W = NT <= 2 ? 16 : 8;
        constexpr int kParts[] = {16, 12, 10, 8, 6, 4, 3, 2, 1};
        const int used = p.E < p.R ? p.E : p.R, mean = (p.R + used - 1) / used;
        const float per_row = (float)p.K * size_of(XDT), per_slice = p.out ? (float)p.N * size_of(ODT) * (Y ? 2 : 1) : 0, a_bytes = 2.0f * p.rank * p.K, b_bytes = p.out ? 2.0f * p.rank * p.N : 0;
        int slices = 1, share = 16;
        float least = 0;
        for (const int rows : kParts) {
            if (rows < 16 && rows >= mean) continue;            // (an adapter's rows in one part, as with sixteen)
            const int held = rows < mean ? rows : mean, parts = rows < mean ? p.R / rows + used / 2 : used;
            for (int n = 1; n <= (p.out ? 8 : 1); ++n) {
                const int rounds = (parts * n + kUnits - 1) / kUnits;
                const float cost = rounds * (96e3f + held * per_row + a_bytes + (held * per_slice + b_bytes) / n);
                if (least == 0 || cost < least) least = cost, slices = n, share = rows;
            }
        }
        if constexpr (NT >= 4) {
            // Long matrices of a high rank, which one block after the other would read whole before it begins with its slice: two launches, each cut into many blocks, the first along
            // the rank.  (One row, 4096 x 4096, rank 64 / 128: a call of 14.4 / 15.1 us, which is the host's, as one launch 19.9 / 35.4.)
            const int parts = p.R / 16 + used;
            if (p.coef && (!p.out || ((long)p.rank * p.K >= 1 << 17 && parts * (p.rank + 15) / 16 <= 2 * kUnits))) {
                AdapterArgs q = p;
                q.out = nullptr, q.y = nullptr;
                if (const int rc = launch_shape<XDT, WDT, WDT, false, 16, 1, 1>(q, 16, 1, s, what)) return rc;
                return p.out ? launch_expand<WDT, ODT, Y, NT>(p, 16, kUnits / parts < 1 ? 1 : kUnits / parts > 32 ? 32 : kUnits / parts, s, what) : (int)MOE_OK;
            }
        }
        return launch_shape<XDT, WDT, ODT, Y, W, 1, NT>(p, share, slices, s, what);
    }
    const long rounds = ((long)p.R + kUnits * (kMost - 8) - 1) / (kUnits * (kMost - 8));
    const int share = (int)((p.R + kUnits * rounds - 1) / (kUnits * rounds));
    if (share <= 29) return launch_shape<XDT, WDT, ODT, Y, 8, 2, NT>(p, share, 1, s, what);
    if constexpr (NT <= 4) {
        if (share <= 45) return launch_shape<XDT, WDT, ODT, Y, 8, 3, NT>(p, share, 1, s, what);
    }
    return launch_shape<XDT, WDT, ODT, Y, 8, kMost / 16, NT>(p, share, 1, s, what);
}

template <int XDT, int WDT, int ODT, bool Y>
static int launch_types(const AdapterArgs &p, hipStream_t s, const char *what)
{
    if (p.rank <= 16) return launch_rank<XDT, WDT, ODT, Y, 1>(p, s, what);
    if (p.rank <= 32) return launch_rank<XDT, WDT, ODT, Y, 2>(p, s, what);
    if (p.rank <= 64) return launch_rank<XDT, WDT, ODT, Y, 4>(p, s, what);
    return launch_rank<XDT, WDT, ODT, Y, 8>(p, s, what);
}

}  // namespace moe
