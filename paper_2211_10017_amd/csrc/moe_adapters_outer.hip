// Gradient of the adapters' matrices: out[e][j] = scale_e sum_r coef[r][j] rows[r], over the rows r of every adapter e.
#include "moe_adapters.h"

namespace moe {

// Chunk `index` of the order adapters, chunks: an adapter has a chunk per `chunk` rows, at least one.  slot: the chunk's place among those of adapters with more than one, -1 for others.
// Every lane computes the same answer; false behind the last one.
__device__ inline bool find_chunk(const int32_t *offsets, int E, int R, int chunk, int index, int *e_out, int *lo_out, int *hi_out, int *slot)
{
    const int lane = threadIdx.x & 63;
    int base = 0, slots = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        int lo = 0, hi = 0;
        if (e0 + lane < E) expert_range(offsets, e0 + lane, R, &lo, &hi);
        const int n = e0 + lane < E ? max((hi - lo + chunk - 1) / chunk, 1) : 0, many = n > 1 ? n : 0;
        const int incl = wave_inclusive_sum(n), incl_many = wave_inclusive_sum(many);
        const uint64_t hit = __ballot(base + incl > index);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            const int i = index - base - __shfl(incl - n, src), before = __shfl(incl_many - many, src);
            const int lo_s = __shfl(lo, src), hi_s = __shfl(hi, src);
            *e_out = e0 + src;
            *lo_out = lo_s + i * chunk, *hi_out = min(hi_s, lo_s + (i + 1) * chunk);
            *slot = __shfl(many, src) ? slots + before + i : -1;
            return true;
        }
        base += __shfl(incl, 63), slots += __shfl(incl_many, 63);
    }
    return false;
}

__device__ inline void store_gradient(void *out, int dtype, size_t at, const float (&v)[4])
{
    auto put = [&](auto d) {
        Raw<decltype(d)::value, 4> r;
        r.set(v);
        r.store(out, at);
    };
    if (dtype == MOE_F32) put(std::integral_constant<int, MOE_F32>{});
    else if (dtype == MOE_F16) put(std::integral_constant<int, MOE_F16>{});
    else put(std::integral_constant<int, MOE_BF16>{});
}

// A wavefront: 64 channels, four neighbouring ones per lane, of up to `chunk` rows of an adapter, 32 rows a step (the products' inner axis).  16-bit rows meet the coefficients as two
// 16-bit terms, three of bf16 where the gradient is fp32 (TERMS); fp16 ones in units of a power of two that grows with them.  fp32 rows and coefficients are multiplied in fp32.
// Two steps' rows are under way at a time, and the places of the next two.  `first`: of the rank, of which a wavefront takes 16 NT at most.
// (16384 rows by 64 adapters of 4096, rank 16, both matrices: 268 MB of rows in 72 us = 3.7 TB/s, one step at a time 84; eight channels a lane, which spill, 73.)
template <int DT, int NT, int TERMS>
__device__ inline void outer_item(const OuterArgs &p, const OuterJob &job, int item, int first)
{
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, rank = p.rank, C = job.C;
    int e, lo, hi, slot;
    if (!find_chunk(p.offsets, p.E, p.R, job.chunk, item / job.ncol, &e, &lo, &hi, &slot)) return;
    lo = __builtin_amdgcn_readfirstlane(lo), hi = __builtin_amdgcn_readfirstlane(hi);
    const bool in = item % job.ncol * 64 + 4 * l < C;
    const int c = min(item % job.ncol * 64 + 4 * l, C - 4);     // (past the end: the last channels again, which are not stored)
    float4_t acc[NT][4] = {};
    int unit = -100;                                            // fp16: the accumulators are in units of 2^unit
    // row i of a lane in a step: the 16-bit products take eight neighbouring ones of a lane, the fp32 ones one of every four
    auto row_of = [&](int step, int i) { return lo + 32 * step + (DT == MOE_F32 ? 4 * i + g : 8 * g + i); };
    Raw<DT, 4> x[2][8];
    float f[2][NT][8];
    int id[2][8];
    auto find = [&](auto s_c, int step) {
        constexpr int B = decltype(s_c)::value;
#pragma unroll
        for (int i = 0; i < 8; ++i) id[B][i] = min(row_of(step, i), hi - 1);
        job.map.find(id[B]);
    };
    auto request = [&](auto s_c, int step) {
        constexpr int B = decltype(s_c)::value;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[B][i].load(job.rows, (size_t)id[B][i] * job.map.stride + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float *at = job.coef + (size_t)min(row_of(step, i), hi - 1) * rank;
#pragma unroll
            for (int n = 0; n < NT; ++n) f[B][n][i] = at[min(first + 16 * n + l, rank - 1)];        // (past the rank: rows of the result that are not stored)
        }
        find(s_c, step + 2);
        requested();
    };
    auto use = [&](auto s_c, int step) {
        constexpr int B = decltype(s_c)::value;
        if (lo + 32 * step + 32 > hi) {                         // rows behind the last: 0, on both sides
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool live = row_of(step, i) < hi;
#pragma unroll
                for (int w = 0; w < Raw<DT, 4>::WORDS; ++w) x[B][i].w[w] = live ? x[B][i].w[w] : 0;
#pragma unroll
                for (int n = 0; n < NT; ++n) f[B][n][i] = live ? f[B][n][i] : 0.0f;
            }
        }
        if constexpr (DT == MOE_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[B][n][i], x[B][i].get(t), acc[n][t], 0, 0, 0);
        } else {
            float back = 1.0f;
            if constexpr (DT == MOE_F16) {
                auto largest = [&](auto finite_c) {
                    float most = 0.0f;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float a = fabsf(f[B][n][i]);
                            most = decltype(finite_c)::value && a == INFINITY ? most : fmaxf(most, a);
                        }
#pragma unroll
                    for (int m = 32; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
                    return most;
                };
                float most = largest(std::false_type{});
                if (most == INFINITY) most = largest(std::true_type{});             // (an infinity is its own rank's alone: the others' numbers need their unit)
                const int ex = split_exponent(most);
                if (ex > unit) {
                    const float down = ex - unit > 126 ? 0.0f : exp2i(unit - ex);       // (past that only what was 0 anyway)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[n][t] *= down;
                    unit = ex;
                }
                back = exp2i(-unit);
            }
            uint2 row[8];
            u32x4_t column[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) row[i] = make_uint2(x[B][i].w[0], x[B][i].w[1]);
            transpose_columns(row, column);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                u32x4_t term[3];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Split<DT> s0(DT == MOE_F16 ? f[B][n][2 * i] * back : f[B][n][2 * i]), s1(DT == MOE_F16 ? f[B][n][2 * i + 1] * back : f[B][n][2 * i + 1]);
                    term[0][i] = s0.hi | (uint32_t)s1.hi << 16, term[1][i] = s0.lo | (uint32_t)s1.lo << 16, term[2][i] = s0.rest | (uint32_t)s1.rest << 16;
                }
#pragma unroll
                for (int i = 0; i < TERMS; ++i)
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[n][t] = product16<DT>(term[i], column[t], acc[n][t]);
            }
        }
        requested();
    };
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    const int steps = (hi - lo + 31) / 32;
    if (steps > 0) {
        find(even, 0), find(odd, 1);
        request(even, 0);
        int t = 0;
        for (; t + 2 < steps; t += 2) request(odd, t + 1), use(even, t), request(even, t + 2), use(odd, t + 1);
        if (t + 1 < steps) request(odd, t + 1), use(even, t), use(odd, t + 1);
        else use(even, t);
    }
    if (!in || slot >= job.slots) return;                       // (no partition makes that many: offsets that are none must not write elsewhere)
    const float s = (job.scale ? job.scale[e] : 1.0f), whole = DT == MOE_F16 ? exp2i(unit) : 1.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = first + 16 * n + 4 * g + i;
            if (j >= rank) continue;
            float v[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = DT == MOE_F16 ? acc[n][t][i] * whole : acc[n][t][i];
            if (slot >= 0) {
                *reinterpret_cast<float4_t *>(job.part + ((size_t)slot * rank + j) * C + c) = float4_t{v[0], v[1], v[2], v[3]};
                continue;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] *= s;
            store_gradient(job.out, p.out_dtype, ((size_t)e * rank + j) * C + c, v);
        }
}

// Up to 32 of the rank are a wavefront's; those that take the same rows for more of it run on the same XCD, one after the other.
template <int DT0, int DT1, int NT, int TERMS>
__global__ __launch_bounds__(64, 3) void adapter_outer_kernel(OuterArgs p)
{
    const int turn = blockIdx.x / kXcds, item = turn / p.turns * kXcds + blockIdx.x % kXcds, first = turn % p.turns * 16 * NT;
    if (item >= p.items) return;
    if (item < p.first) outer_item<DT0, NT, DT0 == MOE_BF16 ? TERMS : 2>(p, p.job[0], item, first);
    else outer_item<DT1, NT, DT1 == MOE_BF16 ? TERMS : 2>(p, p.job[1], item - p.first, first);
}

// Sums of the chunks of adapters that have more than one, in their order.  blockIdx.y: the how manieth such adapter, blockIdx.z: the job.
__global__ __launch_bounds__(256) void adapter_join_kernel(OuterArgs p)
{
    const OuterJob &job = p.job[blockIdx.z];
    const int lane = threadIdx.x & 63;
    const size_t size = (size_t)p.rank * job.C, at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (!job.out || (size_t)blockIdx.x * 1024 >= size) return;
    int seen = 0, slots = 0;
    for (int e0 = 0; e0 < p.E; e0 += 64) {
        int lo = 0, hi = 0;
        if (e0 + lane < p.E) expert_range(p.offsets, e0 + lane, p.R, &lo, &hi);
        const int n = (hi - lo + job.chunk - 1) / job.chunk, many = n > 1 ? n : 0;
        const int incl = wave_inclusive_sum(many), order = wave_inclusive_sum(many ? 1 : 0);
        const uint64_t hit = __ballot(many && seen + order - 1 == (int)blockIdx.y);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            const int chunks = __shfl(many, src), first = slots + __shfl(incl - many, src), e = e0 + src;
            if (at >= size || first + chunks > job.slots) return;
            const float s = job.scale ? job.scale[e] : 1.0f;
            float4_t sum = {};
            const float *from = job.part + (size_t)first * size + at;
            int i = 0;
            for (; i + 8 <= chunks; i += 8) {                   // (eight requested together; added in their order)
                float4_t v[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = *reinterpret_cast<const float4_t *>(from + (size_t)(i + q) * size);
#pragma unroll
                for (int q = 0; q < 8; ++q) sum += v[q];
            }
            for (; i < chunks; ++i) sum += *reinterpret_cast<const float4_t *>(from + (size_t)i * size);
            const float v[4] = {sum[0] * s, sum[1] * s, sum[2] * s, sum[3] * s};
            store_gradient(job.out, p.out_dtype, (size_t)e * size + at, v);
            return;
        }
        seen += __shfl(order, 63), slots += __shfl(incl, 63);
    }
}

int launch_adapter_outer(const OuterArgs &args, int dtype0, int dtype1, hipStream_t s, const char *what)
{
    OuterArgs p = args;
    long blocks[2] = {0, 0};
    size_t most = 0;
    p.join = 0;
    for (int i = 0; i < 2; ++i) {
        OuterJob &j = p.job[i];
        if (!j.out) continue;
        j.ncol = (j.C + 63) / 64;
        blocks[i] = ((long)p.R / j.chunk + p.E) * j.ncol;
        if (p.R > j.chunk) {
            const int many = (p.R - 1) / j.chunk < p.E ? (p.R - 1) / j.chunk : p.E;          // (each has more than `chunk` rows)
            p.join = many > p.join ? many : p.join;
            most = (size_t)p.rank * j.C > most ? (size_t)p.rank * j.C : most;
        }
    }
    if (blocks[0] + blocks[1] == 0) return MOE_OK;
    p.first = (int)blocks[0], p.items = (int)(blocks[0] + blocks[1]), p.turns = p.rank <= 16 ? 1 : (p.rank + 31) / 32;
    const long grid = (blocks[0] + blocks[1] + kXcds - 1) / kXcds * kXcds * p.turns;
    if (grid > 0x3ffffff) return fail(MOE_ERR_UNSUPPORTED, "%s: %ld workgroups exceed one launch", what, grid);
    auto run = [&](auto d0, auto d1) {
        constexpr int D0 = decltype(d0)::value, D1 = decltype(d1)::value;
        auto start = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            const auto kernel = p.out_dtype == MOE_F32 ? &adapter_outer_kernel<D0, D1, NT, 3> : &adapter_outer_kernel<D0, D1, NT, 2>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64), 0, s, p);
            return check_launch(what);
        };
        return p.rank <= 16 ? start(std::integral_constant<int, 1>{}) : start(std::integral_constant<int, 2>{});
    };
    const int rc = with_dtype(dtype1, [&](auto d1) {
        return dtype0 == MOE_F16 ? run(std::integral_constant<int, MOE_F16>{}, d1) : run(std::integral_constant<int, MOE_BF16>{}, d1);
    });
    if (rc != MOE_OK || !p.join) return rc;
    hipLaunchKernelGGL(adapter_join_kernel, dim3((unsigned)((most + 1023) / 1024), (unsigned)p.join, 2), dim3(256), 0, s, p);
    return check_launch(what);
}

}  // namespace moe
