// moe_balance_loss, moe_balance_loss_backward: the router's load-balance loss, its per-expert counts and the gate scales, with the gradient of both.
//
//   p = softmax(logits), c_e = assignments of expert e, A = sum c, N = tokens with an assignment, P_e = sum over those tokens of p_te / N
//   loss = coef E sum_e (c_e / A) P_e,     weight_e = d loss / d p_te = coef E c_e / (A N)
//   dlogits_te = dloss p_te (weight_e - sum_j p_tj weight_j) + the gate scales' part
//
// A token's logits are spread over L lanes of a wavefront, V neighbouring ones per lane and step, so that a lane keeps the sums of its own experts in registers over all
// of its tokens; a block's sums meet in LDS and the blocks' in a second launch, in the order of the blocks: no floating-point atomics, the same bits
// every time.  (A launch of one block does without.)  131072 tokens by 256 experts, two each, fp32: forward 42 us = 3.2 TB/s, the blocks' sums 9.4 us,
// backward 53 us = 5.1 TB/s.  Large batches are bound by both the instructions and the loads of too few wavefronts: of the cycles of a SIMD, which has two of them, instructions
// take 53 % forward and 60 % backward.  Small ones are bound by their launches.
#include <math.h>

#include <type_traits>

#include "moe_ffn_common.h"

namespace moe {

// Blocks, one per compute unit (us, forward with the blocks' sums + backward: 131072 tokens by 256 experts 128 blocks 71 + 94, 256 48 + 54, 512 44 + 51, 1024 59 + 53;
// by 64 49 + 52, 30 + 29, 25 + 21, 28 + 21; 16384 by 64 13.3 + 8.0, 11.3 + 5.6, 12.3 + 5.5, 12.2 + 5.5: the largest batches would gain by two per unit).
constexpr int kBalanceThreads = 512, kBalanceMostBlocks = 256, kBalanceMostExperts = 1024, kBalanceMostK = 8;

struct BalanceArgs {
    const void *logits;         // [T, E]
    const int32_t *idx;         // [T, k]; outside [0, E): no assignment
    int T, E, k, renorm, L;     // L: lanes of a token, a power of two
    float coef;
    float *scale;               // [T, k]
    float *part;                // [blocks, E rounded up to four] sums of p
    int32_t *part_count;        // the same, assignments
    int32_t *part_live;         // [blocks] tokens with an assignment
    float *loss, *prob_mean, *weight;
    int32_t *counts;
    // backward
    const float *dloss, *dscale;
    void *dlogits;
};

template <int DT>
__device__ inline float to_f32(uint32_t bits)
{
    if (DT == MOE_F32) return __uint_as_float(bits);
    if (DT == MOE_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    return __uint_as_float(bits << 16);
}

// FULL: the lanes and steps of a token hold its E logits and nothing besides, as they do for powers of two from eight on.  KM: the most experts of a token (with eight
// for all, a token's scalar work is most of it: 131072 tokens by 256 experts, two each, 4 us more of the forward pass).
// What a lane holds of a token: V neighbouring logits in each of S steps, as they lie in memory, the token's experts, their logits and the gradients of their
// scales.  Requested one token ahead, the experts, which the others' addresses depend on, two.
template <int DT, int V, int S, bool FULL, int KM>
struct TokenLoad {
    static constexpr int W = V == 1 ? 1 : DT == MOE_F32 ? 4 : 2;      // words of a step
    uint32_t raw[S][W], chosen[KM];
    int e[KM];
    float ds[KM];

    __device__ inline void request_experts(const BalanceArgs &a, int t)
    {
#pragma unroll
        for (int j = 0; j < KM; ++j)
            if (j < a.k) e[j] = a.idx[(size_t)t * a.k + j];
    }
    __device__ inline void request(const BalanceArgs &a, int t, int lane_in)
    {
        const uint32_t *z32 = reinterpret_cast<const uint32_t *>(a.logits);
        const uint16_t *z16 = reinterpret_cast<const uint16_t *>(a.logits);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int c = V * (lane_in + a.L * s);
            const size_t at = (size_t)t * a.E + (FULL ? c : min(c, a.E - V));      // (past the end: what the last lane holds, which value() leaves out)
            if constexpr (V == 1) raw[s][0] = DT == MOE_F32 ? z32[at] : z16[at];
            else if constexpr (DT == MOE_F32) {
                const uint4 q = *reinterpret_cast<const uint4 *>(z32 + at);
                raw[s][0] = q.x, raw[s][1] = q.y, raw[s][2] = q.z, raw[s][3] = q.w;
            } else {
                const uint2 q = *reinterpret_cast<const uint2 *>(z16 + at);
                raw[s][0] = q.x, raw[s][1] = q.y;
            }
        }
#pragma unroll
        for (int j = 0; j < KM; ++j) {
            if (j >= a.k) break;
            const size_t at = (size_t)t * a.E + (used(a, j) ? e[j] : 0);
            chosen[j] = DT == MOE_F32 ? z32[at] : z16[at];
            if (a.dscale) ds[j] = a.dscale[(size_t)t * a.k + j];
        }
    }
    __device__ inline bool used(const BalanceArgs &a, int j) const { return e[j] >= 0 && e[j] < a.E; }
    __device__ inline float value(const BalanceArgs &a, int s, int i, int lane_in) const
    {
        if (!FULL && V * (lane_in + a.L * s) >= a.E) return -INFINITY;
        if (V == 1 || DT == MOE_F32) return to_f32<DT>(raw[s][i]);
        return to_f32<DT>(i & 1 ? raw[s][i >> 1] >> 16 : raw[s][i >> 1] & 0xffffu);
    }
};

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

// e^x, x <= 0, in the exponential instruction: off by a unit of its own and by 2^-24 of the argument, 1.2e-6 where e^x = 2e-9.  (expf: both directions of
// 131072 tokens by 256 experts 141 us, a good part of it vector instructions.)
__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// op over the L lanes of a token, in the vector unit's own lane permutations up to sixteen of them.
template <class Op>
__device__ inline float over_lanes(float v, int L, Op op)
{
    auto dpp = [&](auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    using std::integral_constant;
    if (L > 1) v = op(v, dpp(integral_constant<int, 0xb1>{}));        // quad_perm 1,0,3,2
    if (L > 2) v = op(v, dpp(integral_constant<int, 0x4e>{}));        // quad_perm 2,3,0,1
    if (L > 4) v = op(v, dpp(integral_constant<int, 0x141>{}));       // row_half_mirror
    if (L > 8) v = op(v, dpp(integral_constant<int, 0x140>{}));       // row_mirror
    if (L > 16) v = op(v, __shfl_xor(v, 16));
    if (L > 32) v = op(v, __shfl_xor(v, 32));
    return v;
}

// Softmax of a token over its L lanes: p[s][i] inv is that of column V (lane_in + L s) + i, and exp_of(z - base) inv that of any logit z of it.
// A token whose logits are all -infinity has nothing to choose: inv = 0.  (A NaN or +infinity among them makes its p NaN.)
template <int DT, int V, int S, bool FULL, int KM>
__device__ inline void token_softmax(const BalanceArgs &a, const TokenLoad<DT, V, S, FULL, KM> &x, int lane_in, float (&p)[S][V], float &base, float &inv)
{
    float m = -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) p[s][i] = x.value(a, s, i, lane_in), m = fmaxf(m, p[s][i]);
    m = over_lanes(m, a.L, [](float u, float v) { return fmaxf(u, v); });
    base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p[s][i] = exp_of(p[s][i] - base);
            sum += p[s][i];
        }
    sum = over_lanes(sum, a.L, [](float u, float v) { return u + v; });
    inv = sum == 0.0f ? 0.0f : 1.0f / sum;
}

// Gate scales of a token's experts: their p, or, renormalised, a softmax over them alone.  That one starts from the largest logit among them, not among all: the p of experts far
// below a token's best are 0 in 32 bits, their shares of each other are not.  Whether the token has an expert at all.
template <int DT, int V, int S, bool FULL, int KM>
__device__ inline bool gate_scales(const BalanceArgs &a, const TokenLoad<DT, V, S, FULL, KM> &x, bool renorm, float base, float inv, float (&scale)[KM])
{
    float from = base, total = 0.0f;
    bool live = false;
    if (renorm) {
        from = -INFINITY;
#pragma unroll
        for (int j = 0; j < KM; ++j)
            if (j < a.k && x.used(a, j)) from = fmaxf(from, to_f32<DT>(x.chosen[j]));
        if (from == -INFINITY) from = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < KM; ++j) {
        if (j >= a.k) break;
        const bool used = x.used(a, j);
        scale[j] = used ? exp_of(to_f32<DT>(x.chosen[j]) - from) : 0.0f;
        total += scale[j];
        live |= used;
    }
    // (inv - inv: 0, or the NaN of a token that holds one)
    const float factor = !renorm ? inv : (total == 0.0f ? 0.0f : 1.0f / total) + (inv - inv);
#pragma unroll
    for (int j = 0; j < KM; ++j)
        if (j < a.k) scale[j] = x.used(a, j) ? scale[j] * factor : 0.0f;
    return live;
}

// The tokens of a thread's L lanes, one after the other, the next one's loads ahead of the work on this one: f(token, whether it is there, loads).
// (Two tokens a turn, so that what is loaded need not be moved, which would wait for it.)
template <int DT, int V, int S, bool FULL, int KM, class F>
__device__ inline void for_tokens(const BalanceArgs &a, int lane_in, F f)
{
    const int per = blockDim.x / a.L, mine = threadIdx.x / a.L;
    const long step = (long)gridDim.x * per;
    auto at = [&](long t) { return (int)(t < a.T ? t : a.T - 1); };
    if (a.T == 0) return;
    TokenLoad<DT, V, S, FULL, KM> x, y;
    long first = (long)blockIdx.x * per, t = first + mine;         // (the block's first token: its loop ends for all of its threads at once)
    x.request_experts(a, at(t));
    y.request_experts(a, at(t + step));
    x.request(a, at(t), lane_in);
    auto turn = [&](TokenLoad<DT, V, S, FULL, KM> &now, TokenLoad<DT, V, S, FULL, KM> &next) {
        next.request(a, at(t + step), lane_in);
        f(at(t), t < a.T, now);
        now.request_experts(a, at(t + 2 * step));
        first += step, t += step;
    };
    while (first < a.T) {
        turn(x, y);
        if (first >= a.T) break;
        turn(y, x);
    }
}

// What follows from the sums of all tokens: thread q < quads of one block has those of experts 4 q .. 4 q + 3, N the number of tokens with an assignment.
__device__ inline void balance_end(const BalanceArgs &a, const float (&ps)[4], const int (&ns)[4], int q, bool mine, int N)
{
    __shared__ int32_t assigned[16];
    __shared__ float losses[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x / 64;
    int total = mine ? ns[0] + ns[1] + ns[2] + ns[3] : 0;
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o);
    if (lane == 0) assigned[wave] = total;
    __syncthreads();
    int A = 0;
    for (int w = 0; w < waves; ++w) A += assigned[w];
    const float fa = (float)max(A, 1), fn = (float)max(N, 1);
    float loss = 0.0f;
    if (mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 4 * q + i;
            if (c >= a.E) break;
            const float w = a.coef * (float)a.E * ((float)ns[i] / fa), mean = ps[i] / fn;
            loss += w * mean;
            a.counts[c] = ns[i], a.prob_mean[c] = mean, a.weight[c] = w / fn;
        }
    }
    for (int o = 1; o < 64; o <<= 1) loss += __shfl_xor(loss, o);
    if (lane == 0) losses[wave] = loss;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < waves; ++w) loss += losses[w];
    *a.loss = loss;
}

template <int DT, int V, int S, bool FULL, int KM>
__global__ __launch_bounds__(kBalanceThreads) void balance_forward_kernel(BalanceArgs a)
{
    extern __shared__ float sums[];                             // [wavefronts][E]
    __shared__ int32_t cnt[kBalanceMostExperts + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x / 64, L = a.L, lane_in = lane & (L - 1);
    for (int i = tid; i <= a.E; i += blockDim.x) cnt[i] = 0;
    __syncthreads();
    float acc[S][V] = {};
    const bool renorm = a.renorm && a.k > 1;
    for_tokens<DT, V, S, FULL, KM>(a, lane_in, [&](int t, bool here, const TokenLoad<DT, V, S, FULL, KM> &x) {
        float scale[KM], base, inv, p[S][V];
        token_softmax<DT, V, S, FULL, KM>(a, x, lane_in, p, base, inv);
        const bool live = gate_scales<DT, V, S, FULL, KM>(a, x, renorm, base, inv, scale);
        if (here && lane_in == 0) {
            if (live) atomicAdd(&cnt[a.E], 1);
#pragma unroll
            for (int j = 0; j < KM; ++j) {
                if (j >= a.k) break;
                if (x.used(a, j)) atomicAdd(&cnt[x.e[j]], 1);
                a.scale[(size_t)t * a.k + j] = scale[j];
            }
        }
        if (__all(here && live)) {
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[s][i] = fmaf(p[s][i], inv, acc[s][i]);
        } else {                                                // (not by a factor of 0: a pruned token's p may be NaN)
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[s][i] += here && live ? p[s][i] * inv : 0.0f;
        }
    });
    // the lanes of a wavefront that hold the same experts, then the wavefronts
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v = acc[s][i];
            for (int o = L; o < 64; o <<= 1) v += __shfl_xor(v, o);
            const int c = V * (lane_in + L * s) + i;
            if (lane < L && c < a.E) sums[wave * a.E + c] = v;
        }
    __syncthreads();
    const int pitch = (a.E + 3) & ~3;
    if (gridDim.x == 1) {
        float ps[4] = {};
        int ns[4] = {};
        const bool mine = 4 * tid < a.E;                        // (at most 256 threads)
        if (mine)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = 4 * tid + i;
                if (c >= a.E) break;
                for (int w = 0; w < waves; ++w) ps[i] += sums[w * a.E + c];
                ns[i] = cnt[c];
            }
        balance_end(a, ps, ns, tid, mine, cnt[a.E]);
        return;
    }
    for (int c = tid; c < pitch; c += blockDim.x) {
        float v = 0.0f;
        if (c < a.E)
            for (int w = 0; w < waves; ++w) v += sums[w * a.E + c];
        a.part[(size_t)blockIdx.x * pitch + c] = v;
        a.part_count[(size_t)blockIdx.x * pitch + c] = c < a.E ? cnt[c] : 0;
    }
    if (tid == 0) a.part_live[blockIdx.x] = cnt[a.E];
}

// The blocks' sums of every expert, in a fixed order, and what follows from them; one block.  Four experts per thread, and as many strands of blocks
// beside each other as threads allow.
__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceArgs a, int blocks)
{
    __shared__ float4 fs[1024];
    __shared__ int4 is[1024];
    __shared__ int32_t tokens[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pitch = (a.E + 3) & ~3, quads = pitch / 4;
    int cols = 1;
    while (cols < quads) cols <<= 1;                            // (at most 256)
    const int strands = 1024 / cols, strand = tid / cols, q = tid % cols;
    float4 v = make_float4(0, 0, 0, 0);
    int4 n = make_int4(0, 0, 0, 0);
    if (q < quads) {
#pragma unroll 4
        for (int b = strand; b < blocks; b += strands) {
            const float4 f = reinterpret_cast<const float4 *>(a.part + (size_t)b * pitch)[q];
            const int4 i = reinterpret_cast<const int4 *>(a.part_count + (size_t)b * pitch)[q];
            v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
            n.x += i.x, n.y += i.y, n.z += i.z, n.w += i.w;
        }
    }
    int live = tid < blocks ? a.part_live[tid] : 0;             // (at most 256 blocks)
    for (int o = 1; o < 64; o <<= 1) live += __shfl_xor(live, o);
    fs[tid] = v, is[tid] = n;
    if (lane == 0) tokens[wave] = live;
    for (int half = strands / 2; half; half >>= 1) {
        __syncthreads();
        if (strand < half) {
            const float4 f = fs[tid + half * cols];
            const int4 i = is[tid + half * cols];
            v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
            n.x += i.x, n.y += i.y, n.z += i.z, n.w += i.w;
            fs[tid] = v, is[tid] = n;
        }
    }
    __syncthreads();
    int N = 0;
    for (int w = 0; w < 16; ++w) N += tokens[w];
    const float ps[4] = {v.x, v.y, v.z, v.w};
    const int ns[4] = {n.x, n.y, n.z, n.w};
    balance_end(a, ps, ns, q, strand == 0 && q < quads, N);
}

template <int DT, int V, int S, bool FULL, int KM>
__global__ __launch_bounds__(kBalanceThreads) void balance_backward_kernel(BalanceArgs a)
{
    const int lane_in = threadIdx.x & (a.L - 1), L = a.L;
    const float dloss = a.dloss ? *a.dloss : 0.0f;
    float w[S][V];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = V * (lane_in + L * s) + i;
            w[s][i] = c < a.E ? dloss * a.weight[c] : 0.0f;
        }
    const bool renorm = a.renorm && a.k > 1;
    for_tokens<DT, V, S, FULL, KM>(a, lane_in, [&](int t, bool here, const TokenLoad<DT, V, S, FULL, KM> &x) {
        float sc[KM], ds[KM], base, inv, p[S][V];
        token_softmax<DT, V, S, FULL, KM>(a, x, lane_in, p, base, inv);
        const bool live = gate_scales<DT, V, S, FULL, KM>(a, x, renorm, base, inv, sc);
        float mean = 0.0f;                                    // sum_j s_j ds_j
#pragma unroll
        for (int j = 0; j < KM; ++j) {
            if (j >= a.k) break;
            ds[j] = x.used(a, j) && a.dscale ? x.ds[j] : 0.0f;
            mean += sc[j] * ds[j];
        }
        // Renormalised scales are a softmax over the chosen experts: s_j (ds_j - sum_i s_i ds_i), which, as the s_i add up to one, is
        // s_j sum_i s_i (ds_j - ds_i): nothing is lost where the ds are nearly the same.
        float gate[KM];
#pragma unroll
        for (int j = 0; j < KM; ++j) {
            if (j >= a.k) break;
            float d = ds[j];
            if (renorm) {
                d = 0.0f;
#pragma unroll
                for (int i = 0; i < KM; ++i)
                    if (i < a.k) d += sc[i] * (ds[j] - ds[i]);
            }
            gate[j] = sc[j] * d;
        }
        float pw = 0.0f;
#pragma unroll
        for (int q = 0; q < S; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) pw += p[q][i] * w[q][i];
        pw = inv * over_lanes(pw, L, [](float u, float v) { return u + v; });
        const float off = renorm ? pw : pw + mean;            // what every expert's gradient loses, times its p
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int c = V * (lane_in + L * q);
            float g[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                g[i] = p[q][i] * inv * (w[q][i] - off);
#pragma unroll
                for (int j = 0; j < KM; ++j) {
                    if (j >= a.k) break;
                    if (x.e[j] == c + i) g[i] += gate[j];
                }
                if (!live) g[i] = 0.0f;
            }
            if (here && c < a.E) store_logits<DT, V>(a, t, c, g);
        }
    });
}

// Lanes of a token and steps, by E: four neighbouring logits a lane where rows allow it; sixteen lanes, which exchange without LDS, as long as a lane then holds
// no more than four steps.
struct BalanceShape { int V, S, L; };
static BalanceShape balance_shape(int E)
{
    BalanceShape b;
    b.V = E % 4 == 0 ? 4 : 1;
    const int cols = E / b.V;
    b.L = 1;
    while (b.L < cols && (b.L < 16 || (b.L < 64 && b.L * 4 < cols))) b.L <<= 1;
    b.S = 1;
    while (b.S * b.L < cols) b.S <<= 1;
    return b;
}

// Blocks of the forward launch.  Up to four rounds of tokens stay in one block, which then needs no second launch to join the blocks' sums (us, one block / several and that launch:
// two rounds, 128 tokens by 32 experts 7.2 / 9.4, 64 by 256 9.5 / 10.9; four, 256 by 32 9.3 / 9.3, 128 by 61 9.2 / 9.1, 128 by 256 12.2 / 11.2; eight, 512 by 32 13.5 / 9.4, 256 by 256 17.5 / 11.3).
static int balance_blocks(int T, int E)
{
    const long per = kBalanceThreads / balance_shape(E).L, want = T <= 4 * per ? 1 : ((long)T + per - 1) / per;
    return (int)(want < kBalanceMostBlocks ? want : kBalanceMostBlocks);
}

// Calls f(element type, V, S, FULL, KM) as compile-time numbers.
template <class F>
static void with_shape(int dtype, int E, int k, const BalanceShape &b, F f)
{
    auto shapes = [&](auto dt, auto full, auto km) {
        using std::integral_constant;
        if (b.V == 4) {
            if (b.S == 1) f(dt, integral_constant<int, 4>{}, integral_constant<int, 1>{}, full, km);
            else if (b.S == 2) f(dt, integral_constant<int, 4>{}, integral_constant<int, 2>{}, full, km);
            else f(dt, integral_constant<int, 4>{}, integral_constant<int, 4>{}, full, km);
        } else if constexpr (!decltype(full)::value) {
            if (b.S == 1) f(dt, integral_constant<int, 1>{}, integral_constant<int, 1>{}, full, km);
            else if (b.S <= 4) f(dt, integral_constant<int, 1>{}, integral_constant<int, 4>{}, full, km);
            else f(dt, integral_constant<int, 1>{}, integral_constant<int, 16>{}, full, km);
        }
    };
    auto types = [&](auto full, auto km) {
        if (dtype == MOE_F16) shapes(std::integral_constant<int, MOE_F16>{}, full, km);
        else if (dtype == MOE_BF16) shapes(std::integral_constant<int, MOE_BF16>{}, full, km);
        else shapes(std::integral_constant<int, MOE_F32>{}, full, km);
    };
    if (k > 2) types(std::false_type{}, std::integral_constant<int, kBalanceMostK>{});
    else if (E == 4 * b.L * b.S) types(std::true_type{}, std::integral_constant<int, 2>{});
    else types(std::false_type{}, std::integral_constant<int, 2>{});
}

static int check_balance(const char *what, const void *logits, int dtype, const int32_t *idx, int T, int E, int k)
{
    if (T < 0 || E < 1 || k < 1 || k > E) return fail(MOE_ERR_INVALID_ARG, "%s: need T >= 0 and 1 <= k <= E (T=%d E=%d k=%d)", what, T, E, k);
    if (E > kBalanceMostExperts || k > kBalanceMostK) return fail(MOE_ERR_UNSUPPORTED, "%s: E = %d above %d or k = %d above %d", what, E, kBalanceMostExperts, k, kBalanceMostK);
    if ((long)T * k > 0x7fffffffL) return fail(MOE_ERR_INVALID_ARG, "%s: T*k overflows int32", what);
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
    const size_t blocks = balance_blocks(T, E), pitch = round_up(E, 4);
    return blocks == 1 ? 0 : blocks * (2 * pitch * 4 + 4);
}

extern "C" int moe_balance_loss(const void *logits, int dtype, const int32_t *expert_idx, int T, int E, int k, int renormalize, float coef, float *loss,
                                int32_t *counts, float *prob_mean, float *expert_scale, float *weight, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace moe;
    const char *what = "moe_balance_loss";
    if (int rc = check_balance(what, logits, dtype, expert_idx, T, E, k)) return rc;
    if (!loss || !counts || !prob_mean || !weight || (T && !expert_scale)) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    const size_t need = moe_balance_loss_workspace_bytes(T, E);
    if (need && (!workspace || workspace_bytes < need))
        return fail(MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", what, workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned16(workspace)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const BalanceShape b = balance_shape(E);
    const int blocks = balance_blocks(T, E);
    hipStream_t s = as_stream(stream);
    BalanceArgs a{};
    a.logits = logits, a.idx = expert_idx, a.T = T, a.E = E, a.k = k, a.renorm = renormalize, a.L = b.L, a.coef = coef, a.scale = expert_scale;
    const size_t all = (size_t)blocks * round_up(E, 4);
    a.part = (float *)workspace, a.part_count = (int32_t *)workspace + all, a.part_live = (int32_t *)workspace + 2 * all;
    a.loss = loss, a.counts = counts, a.prob_mean = prob_mean, a.weight = weight;
    with_shape(dtype, E, k, b, [&](auto dt, auto v, auto st, auto full, auto km) {
        hipLaunchKernelGGL((balance_forward_kernel<decltype(dt)::value, decltype(v)::value, decltype(st)::value, decltype(full)::value, decltype(km)::value>), dim3(blocks), dim3(kBalanceThreads),
                           kBalanceThreads / 64 * E * 4, s, a);
    });
    if (blocks == 1) return check_launch(what);
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
    with_shape(dtype, E, k, b, [&](auto dt, auto v, auto st, auto full, auto km) {
        hipLaunchKernelGGL((balance_backward_kernel<decltype(dt)::value, decltype(v)::value, decltype(st)::value, decltype(full)::value, decltype(km)::value>), dim3((unsigned)(want < kBalanceMostBlocks ? want : kBalanceMostBlocks)),
                           dim3(kBalanceThreads), 0, as_stream(stream), a);
    });
    return check_launch(what);
}
