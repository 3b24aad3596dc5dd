// moe_adamw, moe_adamw_state: an AdamW step over many tensors, forty in a launch, moments in fp32 or in 8 bits.
//
//   g = grad grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// All in fp32; p is rounded once to its type, and once more into the copy.  In 8 bits m and r = sqrt(v) are e4m3 numbers in units of 2^e, e = floor(log2 amax) - 7 for each
// 32 neighbouring values: the largest then lies in [128, 256) and every rounding stays below e4m3's largest number; values 2^-17 of it and less become 0, but a positive r at least
// the smallest number, 2^-9 units: an r of 0 beside an m that is not would make a step of m / eps.  The root, as its range is half that of v in powers of two.
// The step itself uses m and v as they are before they are rounded to 8 bits.
//
// To the nearest number r cannot follow its average: with b2 = 0.999 it falls by 0.05 % a step at most, half the distance to the next number is 3 to 6 %, so it stays where it is (as does m, with
// b1 = 0.9, up to 1.6 times short of a constant gradient).  RANDOM: up or down by chance, so that the mean of what is held is the number itself, of m and of r, whatever their change in a step.
// r then wanders about its average, by 4 % under constant gradients and 14 % under normal ones, its mean and that of 1 / r move by less than 2 %.
#include <math.h>

#include "moe_rows.h"

namespace moe {

constexpr int kAdamThreads = 256, kAdamChunk = 4096;            // values of a block, four neighbouring ones per thread and step; of small tensors 1024, a step
constexpr int kAdamTensors = 40;                                // of one launch: their table is a kernel argument

struct AdamTensors {
    moe_adamw_tensor t[kAdamTensors];
    int first[kAdamTensors];                                    // the tensor's first block
    int count, chunk;
    float b1, b2, c1, c2, eps, decay, grad_scale;           // c1 = 1 - b1, decay = 1 - lr wd
    float rate, root;                                           // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    double lr, beta1, beta2;
    const int32_t *step;                                        // [1] or null: t on the device, rate and root come from it
    int number;                                                 // t where the host knows it
};

// b^t by squaring, in products alone: the host's bits and the device's are the same, whichever of them knows t.
__host__ __device__ inline double whole_power(double b, int t)
{
    double r = 1.0;
    for (; t; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}
__host__ __device__ inline float step_rate(double lr, double beta1, int t) { return (float)(lr / (1.0 - whole_power(beta1, t))); }
__host__ __device__ inline float step_root(double beta2, int t) { return (float)(1.0 / sqrt(1.0 - whole_power(beta2, t))); }

// 2^e for whole -127 <= e <= 127 (2^-127 is a subnormal number).
__device__ inline float pow2(int e) { return __uint_as_float(e > -127 ? (uint32_t)(e + 127) << 23 : 1u << 22); }

// The largest of the 32 values that eight neighbouring lanes hold.
__device__ inline float max_of_8_lanes(float v)
{
    v = fmaxf(v, __shfl_xor(v, 1));
    v = fmaxf(v, __shfl_xor(v, 2));
    return fmaxf(v, __shfl_xor(v, 4));
}

// Scale byte of a block whose largest magnitude is amax: 255 (not a number) for an infinity or a NaN.
__device__ inline int scale_byte(float amax)
{
    const int e = (int)(__float_as_uint(amax) >> 23);           // (amax >= 0)
    return e == 255 ? 255 : max(e - 134, -127) + 127;
}

__device__ inline float scale_value(int byte) { return byte == 255 ? NAN : pow2(byte - 127); }

// 32 bits for a number of 32: products with odd numbers (the fractions of the golden ratio and of the root of 2), each between shifts that bring the upper half to the lower one.
__device__ inline uint32_t mixed(uint32_t x)
{
    x = (x ^ x >> 16) * 0x9e3779b1u;
    x = (x ^ x >> 15) * 0x6a09e667u;
    return x ^ x >> 16;
}

// a >= 0 to one of the two e4m3 numbers beside it: up where the 20 bits behind the third of the mantissa and 20 random ones together carry.  Numbers below 2^-6, whose steps are all 2^-9, are
// brought into [2^-6, 2^-5), where the steps are the same.
__device__ inline float rounded_by(float a, uint32_t random)
{
    const float up = a < 0x1p-6f ? 0x1p-6f : 0.0f;
    return __uint_as_float((__float_as_uint(a + up) + (random >> 12)) & 0xfff00000u) - up;
}

// Four values in 8 bits.  ROOT: of r = sqrt(v), which stays above 0.  RANDOM: by each value's 32 random bits, of which r takes the upper and m the lower ones (in reverse).
template <bool ROOT, bool RANDOM>
__device__ inline uint32_t encode(const float (&v)[4], int byte, const uint32_t (&random)[4])
{
    if (byte == 255) return 0;
    const float inv = pow2(127 - byte);
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[i] = v[i] * inv;
        if constexpr (RANDOM) q[i] = ROOT ? rounded_by(q[i], random[i]) : copysignf(rounded_by(fabsf(q[i]), __brev(random[i])), q[i]);
        if (ROOT && v[i] > 0.0f) q[i] = fmaxf(q[i], 0x1p-9f);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
}

__device__ inline void decode(uint32_t w, int byte, float (&v)[4])
{
    const float s = scale_value(byte);
    v[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * s, v[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * s;
    v[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * s, v[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * s;
}

// Four neighbouring values, `n` of them there; WIDE: the tensor's buffers are aligned for whole loads.
template <int DT, bool WIDE>
__device__ inline void load4(const void *base, int64_t at, int n, float (&v)[4])
{
    if (WIDE && n == 4) {
        Raw<DT, 4> r;
        r.load(base, (size_t)at);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r.get(i);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? load_one<DT>(base, (size_t)at + i) : 0.0f;
}

template <int DT, bool WIDE>
__device__ inline void store4(void *base, int64_t at, int n, const float (&v)[4])
{
    if (WIDE && n == 4) {
        Raw<DT, 4> r;
        r.set(v);
        r.store(base, (size_t)at);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) store_one<DT>(base, (size_t)at + i, v[i]);
}

template <bool WIDE>
__device__ inline uint32_t load_codes(const uint8_t *base, int64_t at, int n)
{
    if (WIDE && n == 4) return *reinterpret_cast<const uint32_t *>(base + at);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) w |= (uint32_t)base[at + i] << (8 * i);
    return w;
}

template <bool WIDE>
__device__ inline void store_codes(uint8_t *base, int64_t at, int n, uint32_t w)
{
    if (WIDE && n == 4) {
        *reinterpret_cast<uint32_t *>(base + at) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) base[at + i] = (uint8_t)(w >> (8 * i));
}

// Bound by memory: 134 million values with states in 8 bits, bf16 gradients and copies 16.1 bytes each, 405 us = 5.3 TB/s (a call of 417 to the nearest, 419 RANDOM); 25 million with fp32 states 28 bytes each, 139 us = 5.1 TB/s.
// The products and sums of m and v are rounded one by one (no fused multiply-adds): the definition is then the same on every path.
template <int PDT, int GDT, int CDT, int STATES, bool WIDE>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamTensors a)
{
#pragma clang fp contract(off)
    constexpr int BITS = STATES & 0xff;
    constexpr bool RANDOM = (STATES & MOE_ADAMW_RANDOM) != 0;
    __shared__ float from_step[2];
    float rate = a.rate, root = a.root;
    int number = a.number;
    if (a.step) {
        number = max(*a.step, 1);
        if (threadIdx.x == 0) from_step[0] = step_rate(a.lr, a.beta1, number), from_step[1] = step_root(a.beta2, number);
        __syncthreads();
        rate = from_step[0], root = from_step[1];
    }
    int i = 0;
    while (i + 1 < a.count && (int)blockIdx.x >= a.first[i + 1]) ++i;
    const moe_adamw_tensor &t = a.t[i];
    const int64_t start = (int64_t)((int)blockIdx.x - a.first[i]) * a.chunk, end = min(t.n, start + (int64_t)a.chunk);
    // (a value's random bits come from the step's number and its place alone; a block has one upper half of places)
    const uint32_t seed = RANDOM ? mixed((uint32_t)number ^ mixed((uint32_t)(start >> 32))) : 0;
    for (int64_t at = start + threadIdx.x * 4; at < (end + 31) / 32 * 32; at += kAdamThreads * 4) {      // (whole blocks of 32: their eight lanes stay together)
        const int n = (int)min((int64_t)4, max((int64_t)0, end - at));
        float p[4], g[4], m[4], v[4], r[4];
        load4<PDT, WIDE>(t.p, at, n, p);
        load4<GDT, WIDE>(t.g, at, n, g);
        if constexpr (BITS == 8) {
            decode(load_codes<WIDE>((const uint8_t *)t.m, at, n), t.m_scales[at >> 5], m);
            decode(load_codes<WIDE>((const uint8_t *)t.v, at, n), t.v_scales[at >> 5], r);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = r[q] * r[q];
        } else {
            load4<MOE_F32, WIDE>(t.m, at, n, m);
            load4<MOE_F32, WIDE>(t.v, at, n, v);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float h = g[q] * a.grad_scale;
            m[q] = m[q] * a.b1 + h * a.c1;
            v[q] = v[q] * a.b2 + h * h * a.c2;
            r[q] = sqrtf(v[q]);
            p[q] = p[q] * a.decay - rate * m[q] / (r[q] * root + a.eps);
        }
        store4<PDT, WIDE>(t.p, at, n, p);
        if constexpr (CDT >= 0) store4<CDT, WIDE>(t.copy, at, n, p);
        if constexpr (BITS == 8) {
            float ma = 0.0f, ra = 0.0f;
            bool fine = true;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q >= n) m[q] = 0.0f, r[q] = 0.0f;
                ma = fmaxf(ma, fabsf(m[q])), ra = fmaxf(ra, r[q]);
                fine = fine && m[q] == m[q] && r[q] == r[q];                     // (a maximum passes over a NaN)
            }
            if (!fine) ma = ra = INFINITY;
            const int mb = scale_byte(max_of_8_lanes(ma)), rb = scale_byte(max_of_8_lanes(ra));
            uint32_t random[4] = {};
            if constexpr (RANDOM) {
#pragma unroll
                for (int q = 0; q < 4; ++q) random[q] = mixed(((uint32_t)at + q) ^ seed);
            }
            store_codes<WIDE>((uint8_t *)t.m, at, n, encode<false, RANDOM>(m, mb, random));
            store_codes<WIDE>((uint8_t *)t.v, at, n, encode<true, RANDOM>(r, rb, random));
            if ((threadIdx.x & 7) == 0) t.m_scales[at >> 5] = (uint8_t)mb, t.v_scales[at >> 5] = (uint8_t)rb;
        } else {
            store4<MOE_F32, WIDE>(t.m, at, n, m);
            store4<MOE_F32, WIDE>(t.v, at, n, v);
        }
    }
}

// Sixteen values a thread; WIDE: the buffers are aligned for whole loads.  (134 million values to bf16: 85 us = 4.7 TB/s, four a thread 123.)
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void adamw_state_kernel(const uint8_t *codes, const uint8_t *scales, int64_t n, void *out)
{
    for (int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16; at < n; at += (int64_t)gridDim.x * 4096) {
        const int here = (int)min((int64_t)16, n - at), scale = scales[at >> 5];
        if (WIDE && here == 16) {
            const uint4 q = *reinterpret_cast<const uint4 *>(codes + at);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            constexpr int V = DT == MOE_F32 ? 4 : 8;
#pragma unroll
            for (int i = 0; i < 16; i += V) {
                float v[V];
#pragma unroll
                for (int k = 0; k < V; k += 4) {
                    float four[4];
                    decode(w[(i + k) / 4], scale, four);
#pragma unroll
                    for (int t = 0; t < 4; ++t) v[k + t] = four[t];
                }
                Raw<DT, V> r;
                r.set(v);
                r.store(out, (size_t)at + i);
            }
            continue;
        }
        for (int i = 0; i < here; i += 4) {
            const int some = min(4, here - i);
            float v[4];
            decode(load_codes<false>(codes, at + i, some), scale, v);
            store4<DT, false>(out, at + i, some, v);
        }
    }
}

static bool aligned(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// What a step takes; wide: every buffer is aligned for whole loads.
static int check_adamw(const moe_adamw_tensor *tensors, int count, int p_dtype, int g_dtype, int copy_dtype, int state_bits, double lr, double beta1, double beta2, double eps,
                       double weight_decay, double grad_scale, int step, const int32_t *step_ptr, bool *wide_out)
{
    const char *what = "moe_adamw";
    if (count < 0 || (count > 0 && !tensors)) return fail(MOE_ERR_INVALID_ARG, "%s: no tensors", what);
    if (!known_dtype(p_dtype) || !known_dtype(g_dtype) || (copy_dtype != -1 && copy_dtype != MOE_F16 && copy_dtype != MOE_BF16)) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (copy_dtype != -1 && p_dtype != MOE_F32) return fail(MOE_ERR_UNSUPPORTED, "%s: a copy belongs to fp32 parameters", what);
    if (state_bits != 32 && state_bits != 8 && state_bits != (8 | MOE_ADAMW_RANDOM)) return fail(MOE_ERR_UNSUPPORTED, "%s: states of %d bits", what, state_bits);
    if (!step_ptr && step < 1) return fail(MOE_ERR_INVALID_ARG, "%s: steps are counted from 1", what);
    if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1)) return fail(MOE_ERR_INVALID_ARG, "%s: 0 <= beta < 1 required", what);
    if (!(lr >= 0) || !(eps >= 0) || !(weight_decay >= 0) || !isfinite(lr) || !isfinite(eps) || !isfinite(weight_decay) || !isfinite(grad_scale))
        return fail(MOE_ERR_INVALID_ARG, "%s: lr, eps and weight_decay must be finite and at least 0, grad_scale finite", what);
    bool wide = true;
    for (int i = 0; i < count; ++i) {
        const moe_adamw_tensor &t = tensors[i];
        if (t.n < 0) return fail(MOE_ERR_INVALID_ARG, "%s: tensor %d has %lld values", what, i, (long long)t.n);
        if (t.n == 0) continue;
        if (t.n > (int64_t)kAdamChunk << 22) return fail(MOE_ERR_UNSUPPORTED, "%s: tensor %d exceeds one launch", what, i);
        if (!t.p || !t.g || !t.m || !t.v || (state_bits != 32 && (!t.m_scales || !t.v_scales)) || (copy_dtype != -1 && !t.copy))
            return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer in tensor %d", what, i);
        const int state = state_bits == 32 ? 4 : 1;
        if (!aligned(t.p, size_of(p_dtype)) || !aligned(t.g, size_of(g_dtype)) || !aligned(t.m, state) || !aligned(t.v, state) || (copy_dtype != -1 && !aligned(t.copy, 2)))
            return fail(MOE_ERR_INVALID_ARG, "%s: a pointer of tensor %d is not aligned for its type", what, i);
        wide = wide && aligned(t.p, 4 * size_of(p_dtype)) && aligned(t.g, 4 * size_of(g_dtype)) && aligned(t.m, 4 * state) && aligned(t.v, 4 * state)
            && (copy_dtype == -1 || aligned(t.copy, 8));
    }
    *wide_out = wide;
    return MOE_OK;
}

}  // namespace moe

extern "C" int moe_adamw_check(const moe_adamw_tensor *tensors, int count, int p_dtype, int g_dtype, int copy_dtype, int state_bits, double lr, double beta1, double beta2, double eps,
                               double weight_decay, double grad_scale, int step, const int32_t *step_ptr)
{
    bool wide;
    return moe::check_adamw(tensors, count, p_dtype, g_dtype, copy_dtype, state_bits, lr, beta1, beta2, eps, weight_decay, grad_scale, step, step_ptr, &wide);
}

extern "C" int moe_adamw(const moe_adamw_tensor *tensors, int count, int p_dtype, int g_dtype, int copy_dtype, int state_bits, double lr, double beta1, double beta2,
                         double eps, double weight_decay, double grad_scale, int step, const int32_t *step_ptr, void *stream)
{
    using namespace moe;
    const char *what = "moe_adamw";
    bool wide;
    if (const int rc = check_adamw(tensors, count, p_dtype, g_dtype, copy_dtype, state_bits, lr, beta1, beta2, eps, weight_decay, grad_scale, step, step_ptr, &wide)) return rc;
    AdamTensors a;
    a.b1 = (float)beta1, a.b2 = (float)beta2, a.c1 = (float)(1.0 - beta1), a.c2 = (float)(1.0 - beta2), a.eps = (float)eps;
    a.decay = (float)(1.0 - lr * weight_decay), a.grad_scale = (float)grad_scale;
    a.lr = lr, a.beta1 = beta1, a.beta2 = beta2, a.step = step_ptr, a.number = step;
    a.rate = step_ptr ? 0.0f : step_rate(lr, beta1, step), a.root = step_ptr ? 0.0f : step_root(beta2, step);
    int64_t most = 0;
    for (int i = 0; i < count; ++i) most = tensors[i].n > most ? tensors[i].n : most;
    a.chunk = most <= 1 << 20 ? kAdamThreads * 4 : kAdamChunk;      // (two tensors of 32768: 3.8 us, 6.0 in blocks of 4096; 48 of 524288 139 a call, 146)
    int i = 0;
    while (i < count) {
        int blocks = 0;
        a.count = 0;
        for (; i < count && a.count < kAdamTensors; ++i) {
            const int64_t n = tensors[i].n, more = (n + a.chunk - 1) / a.chunk;
            if (n == 0) continue;
            if (blocks + more > 1 << 22) break;
            a.t[a.count] = tensors[i], a.first[a.count++] = blocks;
            blocks += (int)more;
        }
        if (!a.count) break;
        const int rc = with_dtype(p_dtype, [&](auto pd) {
            return with_dtype(g_dtype, [&](auto gd) {
                constexpr int P = decltype(pd)::value, G = decltype(gd)::value;
                auto run = [&](auto cd, auto bits, auto w) {
                    hipLaunchKernelGGL((adamw_kernel<P, G, decltype(cd)::value, decltype(bits)::value, decltype(w)::value>), dim3(blocks), dim3(kAdamThreads), 0, as_stream(stream), a);
                    return check_launch(what);
                };
                auto with_width = [&](auto cd, auto bits) { return wide ? run(cd, bits, std::true_type{}) : run(cd, bits, std::false_type{}); };
                auto with_bits = [&](auto cd) {
                    if (state_bits == 32) return with_width(cd, std::integral_constant<int, 32>{});
                    return state_bits == 8 ? with_width(cd, std::integral_constant<int, 8>{}) : with_width(cd, std::integral_constant<int, 8 | MOE_ADAMW_RANDOM>{});
                };
                if constexpr (P == MOE_F32) {
                    if (copy_dtype == MOE_F16) return with_bits(std::integral_constant<int, MOE_F16>{});
                    if (copy_dtype == MOE_BF16) return with_bits(std::integral_constant<int, MOE_BF16>{});
                }
                return with_bits(std::integral_constant<int, -1>{});
            });
        });
        if (rc != MOE_OK) return rc;
    }
    return MOE_OK;
}

extern "C" int moe_adamw_state(const void *codes, const void *scales, int64_t n, void *out, int out_dtype, void *stream)
{
    using namespace moe;
    const char *what = "moe_adamw_state";
    if (n < 0) return fail(MOE_ERR_INVALID_ARG, "%s: n >= 0 required", what);
    if (!known_dtype(out_dtype)) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (n == 0) return MOE_OK;
    if (!codes || !scales || !out) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned(out, size_of(out_dtype))) return fail(MOE_ERR_INVALID_ARG, "%s: out is not aligned for its type", what);
    const bool wide = aligned(codes, 16) && aligned(out, 16);
    const int64_t blocks = (n + 4095) / 4096;
    return with_dtype(out_dtype, [&](auto d) {
        auto run = [&](auto w) {
            hipLaunchKernelGGL((adamw_state_kernel<decltype(d)::value, decltype(w)::value>), dim3((unsigned)(blocks < 0x40000 ? blocks : 0x40000)), dim3(256), 0, as_stream(stream),
                               (const uint8_t *)codes, (const uint8_t *)scales, n, out);
            return check_launch(what);
        };
        return wide ? run(std::true_type{}) : run(std::false_type{});
    });
}
