// moe_mx4_quantize_rows, moe_mx4_quantize_experts, moe_mx4_dequantize: values to and from the microscaled 4-bit format.
#include <type_traits>

#include "moe_mx4_common.h"

namespace moe {

__device__ inline uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Eight neighbouring values of a row as fp32.
template <int DT>
__device__ inline void load_eight(const void *base, size_t at, float (&v)[8])
{
    if constexpr (DT == MOE_F32) {
        const f32x4_t *q = reinterpret_cast<const f32x4_t *>(reinterpret_cast<const float *>(base) + at);
        const f32x4_t a = q[0], b = q[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
        const u32x4_t w = *reinterpret_cast<const u32x4_t *>(reinterpret_cast<const uint16_t *>(base) + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint16_t b = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
            v[i] = DT == MOE_BF16 ? __uint_as_float((uint32_t)b << 16) : (float)__builtin_bit_cast(_Float16, b);
        }
    }
}

// Sixteen lanes hold 128 values of a row, eight each: the largest magnitude of a block is that of four neighbouring lanes, and every lane of
// the sixteen gets the four scale bytes as the dword that is stored.
__device__ inline uint32_t sixteen_lane_scales(uint32_t amax, uint32_t &byte)
{
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xb1, 0xf, 0xf, true));      // quad_perm 1,0,3,2
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4e, 0xf, 0xf, true));      // quad_perm 2,3,0,1
    byte = mx_scale_byte(amax);
    const int lane = threadIdx.x & 63, quad = (lane >> 2) & 3;
    uint32_t d = byte << (8 * quad);
    d |= __shfl_xor(d, 4);
    d |= __shfl_xor(d, 8);
    return d;
}

// Rows: a wavefront takes four rows by 128 values at a time, sixteen lanes a row, so that loads are whole lines and the scales of a block's
// sixteen rows one 64-byte piece.  Memory-bound: reads K values of a row once, writes 17/32 byte each (16384 rows of 4096, bf16: 34 us = 5.0 TB/s, what a copy reaches).
template <int DT>
__global__ __launch_bounds__(256) void mx4_quantize_rows_kernel(const void *__restrict__ x, int R, int K, long stride, int per,
                                                                uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const int tid = threadIdx.x, part = tid & 15;
    const int G = mx_groups(K), chunks = (G + per - 1) / per;
    const int row = (int)(blockIdx.x / chunks) * 16 + (tid >> 4), g0 = (int)(blockIdx.x % chunks) * per;
    const bool live = row < R;
    for (int g = g0; g < min(g0 + per, G); ++g) {
        const int k = g * kMxGroup + part * 8;
        float v[8] = {};
        if (live && k < K) load_eight<DT>(x, (size_t)row * stride + k, v);
        uint32_t amax = 0, byte;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max(amax, abs_bits(v[i]));
        const uint32_t d = sixteen_lane_scales(amax, byte);
        if (!live) continue;
        if (k < K) *reinterpret_cast<uint32_t *>(codes + (size_t)row * (K / 2) + k / 2) = mx_codes(v, byte);
        if (part == 0) *reinterpret_cast<uint32_t *>(scales + ((size_t)g * R + row) * 4) = d;
    }
}

// Experts: w is [K, N] with N contiguous and a block runs along K: a lane owns two channels and walks down the 32 values of a block, the eight wavefronts of
// a workgroup eight blocks, and the codes go through LDS so that they are stored as whole lines too, eight lanes a channel.  Memory-bound.
// (A lane storing its channel's sixteen bytes at a time: 32 experts of 1024 x 4096 173 us, so 130 = 4.7 TB/s, a channel per lane 135.)
__global__ __launch_bounds__(512) void mx4_quantize_experts_kernel(const float *__restrict__ w, int K, int N, uint8_t *__restrict__ codes,
                                                                   uint8_t *__restrict__ scales)
{
    __shared__ u32x4_t tile[128][9];                                   // (nine: neighbouring channels' blocks start in other banks)
    __shared__ __align__(8) uint8_t bytes[128][8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int blocks = K / kMxBlock, slices = (blocks + 7) / 8, ncol = (N + 127) / 128;
    const int col = (int)(blockIdx.x % ncol), slice = (int)(blockIdx.x / ncol % slices);
    const size_t e = blockIdx.x / ncol / slices;
    const int n = col * 128 + 2 * lane, block = slice * 8 + wave;
    uint32_t byte[2] = {0, 0};
    if (n < N && block < blocks) {
        const float *src = w + (e * K + (size_t)block * kMxBlock) * N + n;
        float2 v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = *reinterpret_cast<const float2 *>(src + (size_t)i * N);
        uint32_t amax[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 32; ++i) amax[0] = max(amax[0], abs_bits(v[i].x)), amax[1] = max(amax[1], abs_bits(v[i].y));
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            byte[s] = mx_scale_byte(amax[s]);
            u32x4_t c;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float t[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] = s ? v[8 * q + i].y : v[8 * q + i].x;
                c[q] = mx_codes(t, byte[s]);
            }
            tile[2 * lane + s][wave] = c;
        }
    }
    bytes[2 * lane][wave] = (uint8_t)byte[0], bytes[2 * lane + 1][wave] = (uint8_t)byte[1];
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int i = half * 64 + (tid >> 3), m = col * 128 + i, b = slice * 8 + (tid & 7);
        if (m < N && b < blocks) *reinterpret_cast<u32x4_t *>(codes + (e * N + m) * (size_t)(K / 2) + (size_t)b * 16) = tile[i][tid & 7];
    }
    const int i = tid & 127, m = col * 128 + i, g = slice * 2 + (tid >> 7);
    if (tid < 256 && m < N && g < mx_groups(K))
        *reinterpret_cast<uint32_t *>(scales + ((e * mx_groups(K) + g) * (size_t)N + m) * 4) = *reinterpret_cast<const uint32_t *>(&bytes[i][4 * (tid >> 7)]);
}

// Codes times scales: eight values a lane, a row's 128 values in sixteen neighbouring lanes.  Memory-bound by what it writes (16384 rows of 4096 to bf16: 30 us = 5.7 TB/s).
template <int DT>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int matrices, int rows,
                                                             int K, void *__restrict__ out)
{
    const int part = threadIdx.x & 15, G = mx_groups(K);
    const int n = (int)(blockIdx.x / G) * 16 + (threadIdx.x >> 4), g = (int)(blockIdx.x % G), k = g * kMxGroup + part * 8;
    if (n >= rows || k >= K) return;
    for (int m = blockIdx.y; m < matrices; m += gridDim.y) {      // (the same for all: no row's matrix has to be found by division)
        const size_t row = (size_t)m * rows + n;
        const uint32_t c = *reinterpret_cast<const uint32_t *>(codes + row * (K / 2) + k / 2);
        const uint32_t byte = scales[(((size_t)m * G + g) * rows + n) * 4 + (part >> 2)];
        const float s = mx_scale_value(byte);
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
        const size_t at = row * K + k;
        if constexpr (DT == MOE_F32) {
            f32x4_t *q = reinterpret_cast<f32x4_t *>(reinterpret_cast<float *>(out) + at);
            q[0] = f32x4_t{p[0][0] * s, p[0][1] * s, p[1][0] * s, p[1][1] * s};
            q[1] = f32x4_t{p[2][0] * s, p[2][1] * s, p[3][0] * s, p[3][1] * s};
        } else {
            u32x4_t w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = p[i][0] * s, hi = p[i][1] * s;
                if (DT == MOE_BF16) w[i] = (uint32_t)to_bf16_rne(lo) | ((uint32_t)to_bf16_rne(hi) << 16);
                else w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16);
            }
            *reinterpret_cast<u32x4_t *>(reinterpret_cast<uint16_t *>(out) + at) = w;
        }
    }
}

constexpr double kMostBlocks = 0xffffff;          // of 256 threads: a launch takes fewer than 2^32 threads

int launch_mx4_quantize_rows(const void *x, int dtype, int R, int K, long stride, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    // Groups of 128 values that a block of sixteen rows takes one after the other: several where there are blocks to spare (us, one / four: fp16, 16384 rows of 4096 32.6 / 30.6, 4096 of
    // 4096 8.5 / 7.9, 16384 of 512 5.5 / 5.3; 1024 of 1024 2.3 / 3.3).  The bound is a little low: 2048 rows of 1024 2.7 / 3.4, 4096 of 1024 3.5 / 4.2.
    const int G = mx_groups(K), per = (long)R * G >= 16384 ? 4 : 1;
    const long blocks = ((long)R + 15) / 16 * ((G + per - 1) / per);
    if (blocks > kMostBlocks) return fail(MOE_ERR_UNSUPPORTED, "moe_mx4_quantize_rows: %ld workgroups exceed one launch", blocks);
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, x, R, K, stride, per, codes, scales); };
    if (dtype == MOE_F16) run(&mx4_quantize_rows_kernel<MOE_F16>);
    else if (dtype == MOE_BF16) run(&mx4_quantize_rows_kernel<MOE_BF16>);
    else run(&mx4_quantize_rows_kernel<MOE_F32>);
    return check_launch("moe_mx4_quantize_rows");
}

}  // namespace moe

extern "C" int moe_mx4_quantize_rows(const void *x, int x_dtype, int R, int K, int64_t x_stride, void *codes, void *scales, void *stream)
{
    using namespace moe;
    const char *what = "moe_mx4_quantize_rows";
    if (R < 0 || K <= 0 || K % 64) return fail(MOE_ERR_INVALID_ARG, "%s: need R >= 0 and K a positive multiple of 64", what);
    if (x_dtype < 0 || x_dtype > 2) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (R == 0) return MOE_OK;                                  // empty buffers may be NULL
    if (!x || !codes || !scales) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(x) || !aligned16(codes) || !aligned16(scales)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    if (x_stride < K || x_stride % (x_dtype == MOE_F32 ? 4 : 8)) return fail(MOE_ERR_INVALID_ARG, "%s: rows of x must be K values or more and 16-byte aligned", what);
    return launch_mx4_quantize_rows(x, x_dtype, R, K, x_stride, (uint8_t *)codes, (uint8_t *)scales, as_stream(stream));
}

extern "C" int moe_mx4_quantize_experts(const float *w, int E, int K, int N, void *codes, void *scales, void *stream)
{
    using namespace moe;
    const char *what = "moe_mx4_quantize_experts";
    if (E < 0 || K <= 0 || N <= 0 || K % 64 || N % 32) return fail(MOE_ERR_INVALID_ARG, "%s: need E >= 0, K %% 64 == 0 and N %% 32 == 0", what);
    if (E == 0) return MOE_OK;
    if (!w || !codes || !scales) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(w) || !aligned16(codes) || !aligned16(scales)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const double blocks = (double)E * (((long)K + 255) / 256) * (((long)N + 127) / 128);
    if (2 * blocks > kMostBlocks) return fail(MOE_ERR_UNSUPPORTED, "%s: %.0f workgroups exceed one launch", what, blocks);
    hipLaunchKernelGGL(mx4_quantize_experts_kernel, dim3((unsigned)blocks), dim3(512), 0, as_stream(stream), w, K, N, (uint8_t *)codes, (uint8_t *)scales);
    return check_launch(what);
}

extern "C" int moe_mx4_dequantize(const void *codes, const void *scales, int matrices, int rows, int K, void *out, int out_dtype, void *stream)
{
    using namespace moe;
    const char *what = "moe_mx4_dequantize";
    if (matrices < 0 || rows < 0 || K <= 0 || K % 64) return fail(MOE_ERR_INVALID_ARG, "%s: need matrices, rows >= 0 and K a positive multiple of 64", what);
    if (out_dtype < 0 || out_dtype > 2) return fail(MOE_ERR_UNSUPPORTED, "%s: unknown dtype", what);
    if (matrices == 0 || rows == 0) return MOE_OK;
    if (!codes || !scales || !out) return fail(MOE_ERR_INVALID_ARG, "%s: NULL pointer", what);
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(out)) return fail(MOE_ERR_INVALID_ARG, "%s: buffers must be 16-byte aligned", what);
    const double blocks = (double)(((long)rows + 15) / 16) * mx_groups(K);
    const int most = matrices < 0x8000 ? matrices : 0x8000;
    if (blocks > kMostBlocks) return fail(MOE_ERR_UNSUPPORTED, "%s: %.0f workgroups exceed one launch", what, blocks);
    auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, (unsigned)most), dim3(256), 0, as_stream(stream), (const uint8_t *)codes, (const uint8_t *)scales, matrices,
                           rows, K, out);
    };
    if (out_dtype == MOE_F16) run(&mx4_dequantize_kernel<MOE_F16>);
    else if (out_dtype == MOE_BF16) run(&mx4_dequantize_kernel<MOE_BF16>);
    else run(&mx4_dequantize_kernel<MOE_F32>);
    return check_launch(what);
}
