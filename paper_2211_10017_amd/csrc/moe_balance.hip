// moe_balance_loss, moe_balance_loss_backward: the router's load-balance loss, its per-expert counts and the gate scales, with the gradient of both.
//
//   p = softmax(logits), c_e = assignments of expert e, A = sum c, N = tokens with an assignment, P_e = sum over those tokens of p_te / N
//   loss = coef E sum_e (c_e / A) P_e,     weight_e = d loss / d p_te = coef E c_e / (A N)
//   dlogits_te = dloss p_te (weight_e - sum_j p_tj weight_j) + the gate scales' part
//
// Both directions are bound by reading the logits (and the backward by writing their gradient), small batches by their launches.  A token's logits are
// spread over L lanes of a wavefront, V neighbouring ones per lane and step, so that a lane keeps the sums of its own experts in registers over all
// of its tokens; a block's sums meet in LDS and the blocks' in a second launch, in the order of the blocks: no floating-point atomics, the same bits
// every time.  (A launch of one block does both.)
#include <math.h>

#include <type_traits>

#include "moe_ffn_common.h"

namespace moe {

constexpr int kBalanceThreads = 512, kBalanceMostBlocks = 256, kBalanceMostExperts = 1024, kBalanceMostK = 8;

struct BalanceArgs {
    const void *logits;         // [T, E]
    const int32_t *idx;         // [T, k]; outside [0, E): no assignment
    int T, E, k, renorm, L;     // L: lanes of a token, a power of two
    float coef;
    float *scale;               // [T, k]
    float *part;                // [blocks, E] sums of p
    int32_t *part_count;        // [blocks, E + 1]: assignments, and tokens with one
    float *loss, *prob_mean, *weight;
    int32_t *counts;
    // backward
    const float *dloss, *dscale;
    void *dlogits;
};

// V neighbouring logits at column c of token t as fp32; -infinity past the end.
template <int DT, int V>
__device__ inline void load_logits(const BalanceArgs &a, int t, int c, float (&v)[V])
{
    const size_t at = (size_t)t * a.E + c;
    if constexpr (V == 1) {
        if constexpr (DT == MOE_F32) v[0] = reinterpret_cast<const float *>(a.logits)[at];
        else if constexpr (DT == MOE_F16) v[0] = (float)reinterpret_cast<const _Float16 *>(a.logits)[at];
        else v[0] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(a.logits)[at] << 16);
    } else if constexpr (DT == MOE_F32) {
        const float4 q = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(a.logits) + at);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
        const uint2 q = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(a.logits) + at);
        const uint16_t b[4] = {(uint16_t)q.x, (uint16_t)(q.x >> 16), (uint16_t)q.y, (uint16_t)(q.y >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = DT == MOE_BF16 ? __uint_as_float((uint32_t)b[i] << 16) : (float)__builtin_bit_cast(_Float16, b[i]);
    }
}

template <int DT, int V>
__device__ inline void store_logits(const BalanceArgs &a, int t, int c, const float (&v)[V])
{
    const size_t at = (size_t)t * a.E + c;
    uint16_t b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = DT == MOE_BF16 ? to_bf16_rne(v[i]) : __builtin_bit_cast(uint16_t, (_Float16)v[i]);
    if constexpr (V == 1) {
        if constexpr (DT == MOE_F32) reinterpret_cast<float *>(a.dlogits)[at] = v[0];
        else reinterpret_cast<uint16_t *>(a.dlogits)[at] = b[0];
    } else if constexpr (DT == MOE_F32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(a.dlogits) + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(a.dlogits) + at) = make_uint2(b[0] | (uint32_t)b[1] << 16, b[2] | (uint32_t)b[3] << 16);
}

__device__ inline float lanes_max(float v, int L)
{
    for (int o = 1; o < L; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ inline float lanes_sum(float v, int L)
{
    for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o);
    return v;
}

// Softmax of a token over its L lanes: p[s][i] of column V (lane_in + L s) + i.  A token whose logits are all -infinity has nothing to choose: p = 0.
// (A NaN or +infinity among them makes its p NaN.)
template <int DT, int V, int S>
__device__ inline void token_softmax(const BalanceArgs &a, int t, int lane_in, float (&p)[S][V])
{
    float m = -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int c = V * (lane_in + a.L * s);
#pragma unroll
        for (int i = 0; i < V; ++i) p[s][i] = -INFINITY;
        if (c < a.E) load_logits<DT, V>(a, t, c, p[s]);
#pragma unroll
        for (int i = 0; i < V; ++i) m = fmaxf(m, p[s][i]);
    }
    m = lanes_max(m, a.L);
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p[s][i] = expf(p[s][i] - base);
            sum += p[s][i];
        }
    sum = lanes_sum(sum, a.L);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) p[s][i] *= inv;
}

// p of expert e, which one of the token's lanes holds, for all of them.
template <int V, int S>
__device__ inline float of_expert(const float (&p)[S][V], int e, int lane_in, int L)
{
    const int lane = threadIdx.x & 63, col = e / V, owner = col % L;
    float mine = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (s * L + lane_in == col && i == e % V) mine = p[s][i];
    return __shfl(mine, (lane & ~(L - 1)) + owner);
}

template <int DT, int V, int S>
__global__ __launch_bounds__(kBalanceThreads) void balance_forward_kernel(BalanceArgs a)
{
    __shared__ float sums[kBalanceThreads / 64][kBalanceMostExperts];
    __shared__ int32_t cnt[kBalanceMostExperts + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, L = a.L, lane_in = lane & (L - 1);
    for (int i = tid; i <= a.E; i += kBalanceThreads) cnt[i] = 0;
    __syncthreads();
    float acc[S][V] = {};
    const int per = kBalanceThreads / L;                       // tokens of a block at a time
    for (long t0 = (long)blockIdx.x * per; t0 < a.T; t0 += (long)gridDim.x * per) {
        const bool here = t0 + tid / L < a.T;
        const int t = here ? (int)(t0 + tid / L) : a.T - 1;
        float p[S][V];
        token_softmax<DT, V, S>(a, t, lane_in, p);
        bool live = false;
        float chosen[kBalanceMostK], total = 0.0f;
#pragma unroll
        for (int j = 0; j < kBalanceMostK; ++j) {
            if (j >= a.k) break;
            const int e = a.idx[(size_t)t * a.k + j];
            const bool used = e >= 0 && e < a.E;
            const float v = of_expert<V, S>(p, used ? e : 0, lane_in, L);
            chosen[j] = used ? v : 0.0f;
            total += chosen[j];
            live |= used;
            if (here && used && lane_in == 0) atomicAdd(&cnt[e], 1);
        }
        if (here && live && lane_in == 0) atomicAdd(&cnt[a.E], 1);
        const float div = a.renorm && a.k > 1 ? (total != 0.0f ? total : 1.0f) : 1.0f;
#pragma unroll
        for (int j = 0; j < kBalanceMostK; ++j) {
            if (j >= a.k) break;
            if (here && lane_in == 0) a.scale[(size_t)t * a.k + j] = chosen[j] / div;
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[s][i] += here && live ? p[s][i] : 0.0f;
    }
    // the lanes of a wavefront that hold the same experts, then the wavefronts
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v = acc[s][i];
            for (int o = L; o < 64; o <<= 1) v += __shfl_xor(v, o);
            const int c = V * (lane_in + L * s) + i;
            if (lane < L && c < a.E) sums[wave][c] = v;
        }
    __syncthreads();
    for (int c = tid; c <= a.E; c += kBalanceThreads) {
        if (c < a.E) {
            float v = 0.0f;
            for (int w = 0; w < kBalanceThreads / 64; ++w) v += sums[w][c];
            a.part[(size_t)blockIdx.x * a.E + c] = v;
        }
        a.part_count[(size_t)blockIdx.x * (a.E + 1) + c] = cnt[c];
    }
}

// The blocks' sums of an expert, in their order, and what follows from them; one block.
__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceArgs a, int blocks)
{
    __shared__ float fs[1024];
    __shared__ int32_t is[1024];
    __shared__ float pc[kBalanceMostExperts];
    __shared__ int32_t cc[kBalanceMostExperts + 1];
    const int tid = threadIdx.x;
    // one expert per thread, in as many strands of blocks as threads allow
    int cols = 1;
    while (cols < a.E + 1 && cols < 1024) cols <<= 1;
    const int strands = 1024 / cols, strand = tid / cols;
    for (int c0 = 0; c0 <= a.E; c0 += cols) {
        const int c = c0 + tid % cols;
        float v = 0.0f;
        int32_t n = 0;
        if (c <= a.E)
            for (int b = strand; b < blocks; b += strands) {
                if (c < a.E) v += a.part[(size_t)b * a.E + c];
                n += a.part_count[(size_t)b * (a.E + 1) + c];
            }
        fs[tid] = v, is[tid] = n;
        __syncthreads();
        if (strand == 0 && c <= a.E) {
            for (int s = 1; s < strands; ++s) v += fs[s * cols + tid], n += is[s * cols + tid];
            if (c < a.E) pc[c] = v;
            cc[c] = n;
        }
        __syncthreads();
    }
    int32_t total = 0;
    for (int c = tid; c < a.E; c += 1024) total += cc[c];
    is[tid] = total;
    __syncthreads();
    for (int o = 512; o; o >>= 1) {
        if (tid < o) is[tid] += is[tid + o];
        __syncthreads();
    }
    const float A = (float)max(is[0], 1), N = (float)max(cc[a.E], 1);
    float loss = 0.0f;
    for (int c = tid; c < a.E; c += 1024) {
        const float w = a.coef * (float)a.E * ((float)cc[c] / A);
        loss += w * (pc[c] / N);
        a.counts[c] = cc[c], a.prob_mean[c] = pc[c] / N, a.weight[c] = w / N;
    }
    fs[tid] = loss;
    __syncthreads();
    for (int o = 512; o; o >>= 1) {
        if (tid < o) fs[tid] += fs[tid + o];
        __syncthreads();
    }
    if (tid == 0) *a.loss = fs[0];
}

template <int DT, int V, int S>
__global__ __launch_bounds__(kBalanceThreads) void balance_backward_kernel(BalanceArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, L = a.L, lane_in = lane & (L - 1);
    const float dloss = a.dloss ? *a.dloss : 0.0f;
    float w[S][V];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = V * (lane_in + L * s) + i;
            w[s][i] = c < a.E ? dloss * a.weight[c] : 0.0f;
        }
    const int per = kBalanceThreads / L;
    for (long t0 = (long)blockIdx.x * per; t0 < a.T; t0 += (long)gridDim.x * per) {
        const bool here = t0 + tid / L < a.T;
        const int t = here ? (int)(t0 + tid / L) : a.T - 1;
        float p[S][V];
        token_softmax<DT, V, S>(a, t, lane_in, p);
        int e[kBalanceMostK];
        float s[kBalanceMostK], ds[kBalanceMostK], total = 0.0f;
        bool live = false;
#pragma unroll
        for (int j = 0; j < kBalanceMostK; ++j) {
            if (j >= a.k) break;
            e[j] = a.idx[(size_t)t * a.k + j];
            const bool used = e[j] >= 0 && e[j] < a.E;
            if (!used) e[j] = -1;
            const float v = of_expert<V, S>(p, used ? e[j] : 0, lane_in, L);
            s[j] = used ? v : 0.0f;
            ds[j] = used && a.dscale ? a.dscale[(size_t)t * a.k + j] : 0.0f;
            total += s[j];
            live |= used;
        }
        const bool renorm = a.renorm && a.k > 1;
        const float div = renorm && total != 0.0f ? total : 1.0f;
        float mean = 0.0f;                                    // sum_j s_j ds_j
#pragma unroll
        for (int j = 0; j < kBalanceMostK; ++j) {
            if (j >= a.k) break;
            s[j] /= div;
            mean += s[j] * ds[j];
        }
        // Renormalised scales are a softmax over the chosen experts: s_j (ds_j - sum_i s_i ds_i), which, as the s_i add up to one, is
        // s_j sum_i s_i (ds_j - ds_i): nothing is lost where the ds are nearly the same.
        float gate[kBalanceMostK];
#pragma unroll
        for (int j = 0; j < kBalanceMostK; ++j) {
            if (j >= a.k) break;
            float d = ds[j];
            if (renorm) {
                d = 0.0f;
#pragma unroll
                for (int i = 0; i < kBalanceMostK; ++i) {
                    if (i >= a.k) break;
                    d += s[i] * (ds[j] - ds[i]);
                }
            }
            gate[j] = s[j] * d;
        }
        float pw = 0.0f;
#pragma unroll
        for (int q = 0; q < S; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) pw += p[q][i] * w[q][i];
        pw = lanes_sum(pw, L);
        const float off = renorm ? pw : pw + mean;            // what every expert's gradient loses, times its p
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int c = V * (lane_in + L * q);
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                g[i] = p[q][i] * (w[q][i] - off);
#pragma unroll
                for (int j = 0; j < kBalanceMostK; ++j) {
                    if (j >= a.k) break;
                    if (e[j] == c + i) g[i] += gate[j];
                }
                if (!live) g[i] = 0.0f;
            }
            if (here && c < a.E) store_logits<DT, V>(a, t, c, g);
        }
    }
}

// Lanes of a token and steps, by E: four neighbouring logits a lane where rows allow it.
struct BalanceShape { int V, S, L; };
static BalanceShape balance_shape(int E)
{
    BalanceShape b;
    b.V = E % 4 == 0 ? 4 : 1;
    const int cols = E / b.V;
    b.L = 1;
    while (b.L < cols && b.L < 64) b.L <<= 1;
    b.S = 1;
    while (b.S * b.L < cols) b.S <<= 1;
    return b;
}

static int balance_blocks(int T, int L)
{
    const long per = kBalanceThreads / L, want = ((long)T + per - 1) / per;
    return (int)(want < kBalanceMostBlocks ? want : kBalanceMostBlocks);
}

// Calls f(element type, V, S) as compile-time numbers.
template <class F>
static void with_shape(int dtype, const BalanceShape &b, F f)
{
    auto steps = [&](auto dt) {
        auto go = [&](auto v, auto s) { f(dt, v, s); };
        using std::integral_constant;
        if (b.V == 4) {
            if (b.S == 1) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
            else if (b.S == 2) go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
            else go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
        } else {
            if (b.S == 1) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
            else if (b.S == 2) go(integral_constant<int, 1>{}, integral_constant<int, 2>{});
            else if (b.S == 4) go(integral_constant<int, 1>{}, integral_constant<int, 4>{});
            else if (b.S == 8) go(integral_constant<int, 1>{}, integral_constant<int, 8>{});
            else go(integral_constant<int, 1>{}, integral_constant<int, 16>{});
        }
    };
    if (dtype == MOE_F16) steps(std::integral_constant<int, MOE_F16>{});
    else if (dtype == MOE_BF16) steps(std::integral_constant<int, MOE_BF16>{});
    else steps(std::integral_constant<int, MOE_F32>{});
}

static int check_balance(const char *what, const void *logits, int dtype, const int32_t *idx, int T, int E, int k)
{
    if (T < 0 || E < 1 || k < 1 || k > E) return fail(MOE_ERR_INVALID_ARG, "%s: need T >= 0 and 1 <= k <= E (T=%d E=%d k=%d)", what, T, E, k);
    if (E > kBalanceMostExperts || k > kBalanceMostK) return fail(MOE_ERR_UNSUPPORTED, "%s: E = %d above %d or k = %d above %d", what, E, kBalanceMostExperts, k, kBalanceMostK);
    if (dtype < 0 || dtype > 2) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (T && (!logits || !idx)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(logits)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    return MOE_OK;
}

}  // namespace moe

extern "C" size_t moe_balance_loss_workspace_bytes(int T, int E)
{
    using namespace moe;
    if (T < 0 || E < 1 || E > kBalanceMostExperts) return 0;
    const size_t blocks = balance_blocks(T, balance_shape(E).L);
    return round_up(blocks * E * 4, 16) + blocks * (E + 1) * 4 + 16;
}

extern "C" int moe_balance_loss(const void *logits, int dtype, const int32_t *expert_idx, int T, int E, int k, int renormalize, float coef, float *loss,
                                int32_t *counts, float *prob_mean, float *expert_scale, float *weight, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace moe;
    const char *what = "moe_balance_loss";
    if (int rc = check_balance(what, logits, dtype, expert_idx, T, E, k)) return rc;
    if (!loss || !counts || !prob_mean || !weight || (T && !expert_scale)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    const size_t need = moe_balance_loss_workspace_bytes(T, E);
    if (!workspace || workspace_bytes < need) return fail(MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", what, workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned16(workspace)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const BalanceShape b = balance_shape(E);
    const int blocks = balance_blocks(T, b.L);
    hipStream_t s = as_stream(stream);
    BalanceArgs a{};
    a.logits = logits, a.idx = expert_idx, a.T = T, a.E = E, a.k = k, a.renorm = renormalize, a.L = b.L, a.coef = coef, a.scale = expert_scale;
    a.part = (float *)workspace, a.part_count = (int32_t *)((uint8_t *)workspace + round_up((size_t)blocks * E * 4, 16));
    a.loss = loss, a.counts = counts, a.prob_mean = prob_mean, a.weight = weight;
    if (blocks)
        with_shape(dtype, b, [&](auto dt, auto v, auto st) {
            hipLaunchKernelGGL((balance_forward_kernel<decltype(dt)::value, decltype(v)::value, decltype(st)::value>), dim3(blocks), dim3(kBalanceThreads), 0, s, a);
        });
    if (int rc = check_launch(what)) return rc;
    hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(1024), 0, s, a, blocks);
    return check_launch(what);
}

extern "C" int moe_balance_loss_backward(const void *logits, int dtype, const int32_t *expert_idx, int T, int E, int k, int renormalize, const float *weight,
                                         const float *dloss, const float *dscale, void *dlogits, void *stream)
{
    using namespace moe;
    const char *what = "moe_balance_loss_backward";
    if (int rc = check_balance(what, logits, dtype, expert_idx, T, E, k)) return rc;
    if (T == 0) return MOE_OK;
    if (!weight || !dlogits) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(dlogits)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const BalanceShape b = balance_shape(E);
    const long want = ((long)T * b.L + kBalanceThreads - 1) / kBalanceThreads;
    BalanceArgs a{};
    a.logits = logits, a.idx = expert_idx, a.T = T, a.E = E, a.k = k, a.renorm = renormalize, a.L = b.L;
    a.weight = const_cast<float *>(weight), a.dloss = dloss, a.dscale = dscale, a.dlogits = dlogits;
    with_shape(dtype, b, [&](auto dt, auto v, auto st) {
        hipLaunchKernelGGL((balance_backward_kernel<decltype(dt)::value, decltype(v)::value, decltype(st)::value>), dim3((unsigned)(want < 2048 ? want : 2048)),
                           dim3(kBalanceThreads), 0, as_stream(stream), a);
    });
    return check_launch(what);
}
