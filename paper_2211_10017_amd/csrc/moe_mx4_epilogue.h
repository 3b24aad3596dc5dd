// The end of a 32-channel by 32-row tile of the 4-bit grouped product.
#pragma once

#include "moe_mx4_common.h"

namespace moe {

// Accumulator of one tile: weights are the matrix instruction's first operand, so a lane holds one row (r = lane & 31) and, with h = lane >> 5, the
// channels 8 q + 4 h + i, q, i = 0..3, of the slab: a block of 32 channels of a row is in two lanes, and quantising the result for the next
// product takes one exchange between them.

// Bias and activation.
__device__ __forceinline__ void mx_finish(const MxArgs &p, const float16_t &acc, int e, int n0, float (&v)[16])
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = acc[i];
    if (p.bias) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x2_t b = *reinterpret_cast<const u32x2_t *>(p.bias + (size_t)e * p.N + n0 + 8 * q + 4 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * q + i] += (float)__builtin_bit_cast(_Float16, (uint16_t)(b[i >> 1] >> (16 * (i & 1))));
        }
    }
    if (p.act == MOE_ACT_RELU) {            // (not fmaxf, which would make a 0 of a NaN, and numbers of a row that holds one)
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];
    } else if (p.act == MOE_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = gelu(v[i]);
    }
}

// The slab as 4-bit codes: of its sixteen bytes lane h gets bytes 8 h .. 8 h + 7.
__device__ __forceinline__ u32x2_t mx_quantize_slab(const float (&v)[16], uint32_t &byte)
{
    const int h = (threadIdx.x & 63) >> 5;
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
    byte = mx_scale_byte(amax);
    uint32_t c[2];                                          // the lane's codes: 16 bits per q
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const float w[8] = {v[8 * t], v[8 * t + 1], v[8 * t + 2], v[8 * t + 3], v[8 * t + 4], v[8 * t + 5], v[8 * t + 6], v[8 * t + 7]};
        c[t] = mx_codes(w, byte);
    }
    // lane h keeps q = 2 h and 2 h + 1 (16 channels, 8 bytes) and gives the other lane its half of the others
    const uint32_t give = h ? c[0] : c[1], keep = h ? c[1] : c[0], got = __shfl_xor((int)give, 32);
    const uint32_t lo = h ? got : keep, hi = h ? keep : got;            // channels 8 q + 0..3 and 8 q + 4..7
    return u32x2_t{(lo & 0xffffu) | (hi << 16), (lo >> 16) | (hi & 0xffff0000u)};
}

__device__ __forceinline__ void mx_store_scale(const MxArgs &p, int n0, int row, uint32_t byte)
{
    p.out_scales[((size_t)(n0 / kMxGroup) * p.R + row) * 4 + (n0 / 32) % 4] = (uint8_t)byte;
}

// Four neighbouring channels in 16 bits.
template <int OUT>
__device__ __forceinline__ u32x2_t mx_pack16(const float *v)
{
    uint16_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = OUT == MOE_BF16 ? to_bf16_rne(v[i]) : __builtin_bit_cast(uint16_t, (_Float16)v[i]);
    return u32x2_t{(uint32_t)b[0] | ((uint32_t)b[1] << 16), (uint32_t)b[2] | ((uint32_t)b[3] << 16)};
}

// One tile by itself.  OUT: MOE_F16, MOE_BF16, MOE_F32, or -1: the 4-bit format.
template <int OUT>
__device__ __forceinline__ void mx_store_tile(const MxArgs &p, const float16_t &acc, int e, int n0, int row, bool live)
{
    const int h = (threadIdx.x & 63) >> 5;
    float v[16];
    mx_finish(p, acc, e, n0, v);
    if constexpr (OUT < 0) {
        uint32_t byte;
        const u32x2_t d = mx_quantize_slab(v, byte);
        if (!live) return;
        *reinterpret_cast<u32x2_t *>(reinterpret_cast<uint8_t *>(p.out) + (size_t)row * (p.N / 2) + n0 / 2 + 8 * h) = d;
        if (h == 0) mx_store_scale(p, n0, row, byte);
    } else if constexpr (OUT == MOE_F32) {
        if (!live) return;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4_t *>(reinterpret_cast<float *>(p.out) + (size_t)row * p.N + n0 + 8 * q + 4 * h) =
                f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    } else {
        if (!live) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<u32x2_t *>(reinterpret_cast<uint16_t *>(p.out) + (size_t)row * p.N + n0 + 8 * q + 4 * h) = mx_pack16<OUT>(v + 4 * q);
    }
}

// Two tiles of the same rows and neighbouring slabs, by way of `patch` (kMxPatch<OUT> bytes of LDS of the wavefront's own): rows leave as whole pieces of 64 channels,
// 16 bytes a lane.  (Eight bytes a lane straight from the accumulators, 4096 tokens, two of 128 experts of 2048 x 8192: 304 us of which the stores are 64.)
template <int OUT>
constexpr int kMxPatch = OUT < 0 ? 0 : 32 * ((OUT == MOE_F32 ? 256 : 128) + 16);

template <int OUT>
__device__ __forceinline__ void mx_store_pair(const MxArgs &p, const float16_t &acc0, const float16_t &acc1, int e, int n0, int row0, int rows, uint8_t *patch)
{
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const bool both = n0 + 32 < p.N;
    if constexpr (OUT < 0) {
        float v[16];
        uint32_t byte[2];
        u32x2_t d[2];
        mx_finish(p, acc0, e, n0, v);
        d[0] = mx_quantize_slab(v, byte[0]);
        mx_finish(p, acc1, e, both ? n0 + 32 : n0, v);
        d[1] = mx_quantize_slab(v, byte[1]);
        // lane h takes all of slab h
        const uint32_t g0 = __shfl_xor((int)(h ? d[0][0] : d[1][0]), 32), g1 = __shfl_xor((int)(h ? d[0][1] : d[1][1]), 32);
        const u32x4_t w = h ? u32x4_t{g0, g1, d[1][0], d[1][1]} : u32x4_t{d[0][0], d[0][1], g0, g1};
        if (r >= rows || (h && !both)) return;
        *reinterpret_cast<u32x4_t *>(reinterpret_cast<uint8_t *>(p.out) + (size_t)(row0 + r) * (p.N / 2) + n0 / 2 + 16 * h) = w;
        mx_store_scale(p, n0 + 32 * h, row0 + r, h ? byte[1] : byte[0]);
    } else {
        constexpr int B = OUT == MOE_F32 ? 4 : 2, PITCH = 64 * B + 16, LANES = 64 * B / 16, ROWS = 64 / LANES;      // bytes of a channel, lanes of a row, rows of a store
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float v[16];
            mx_finish(p, s ? acc1 : acc0, e, s && both ? n0 + 32 : n0, v);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint8_t *at = patch + r * PITCH + (32 * s + 8 * q + 4 * h) * B;
                if constexpr (OUT == MOE_F32) *reinterpret_cast<f32x4_t *>(at) = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                else *reinterpret_cast<u32x2_t *>(at) = mx_pack16<OUT>(v + 4 * q);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int piece = lane % LANES;
        const bool here = both || piece < LANES / 2;
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) {
            const int row = i * ROWS + lane / LANES;
            if (here && row < rows)
                *reinterpret_cast<u32x4_t *>(reinterpret_cast<uint8_t *>(p.out) + ((size_t)(row0 + row) * p.N + n0) * B + piece * 16) =
                    *reinterpret_cast<const u32x4_t *>(patch + row * PITCH + piece * 16);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace moe
