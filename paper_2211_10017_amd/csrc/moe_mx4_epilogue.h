// The end of a 32-channel by 32-row tile of the 4-bit grouped product.
#pragma once

#include "moe_mx4_common.h"

namespace moe {

// Accumulator of one tile: weights are the matrix instruction's first operand, so a lane holds one row (lane & 31) and, with h = lane >> 5, the
// channels 8 q + 4 h + i, q, i = 0..3, of the slab: a block of 32 channels of a row is in two lanes, and quantising the result for the next
// product takes one exchange between them.
template <int OUT>      // MOE_F16, MOE_BF16, MOE_F32, or -1: the 4-bit format
__device__ __forceinline__ void mx_store_tile(const MxArgs &p, const float16_t &acc, int e, int n0, int row, bool live)
{
    const int lane = threadIdx.x & 63, h = lane >> 5;
    float v[16];
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
    if constexpr (OUT < 0) {
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
        const uint32_t byte = mx_scale_byte(amax);
        uint32_t c[2];                                          // the lane's codes: 16 bits per q
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float w[8] = {v[8 * t], v[8 * t + 1], v[8 * t + 2], v[8 * t + 3], v[8 * t + 4], v[8 * t + 5], v[8 * t + 6], v[8 * t + 7]};
            c[t] = mx_codes(w, byte);
        }
        // lane h keeps q = 2 h and 2 h + 1 (16 channels, 8 bytes) and gives the other lane its half of the others
        const uint32_t give = h ? c[0] : c[1], keep = h ? c[1] : c[0], got = __shfl_xor((int)give, 32);
        const uint32_t lo = h ? got : keep, hi = h ? keep : got;            // channels 8 q + 0..3 and 8 q + 4..7
        const u32x2_t d = {(lo & 0xffffu) | (hi << 16), (lo >> 16) | (hi & 0xffff0000u)};
        if (!live) return;
        *reinterpret_cast<u32x2_t *>(reinterpret_cast<uint8_t *>(p.out) + (size_t)row * (p.N / 2) + n0 / 2 + 8 * h) = d;
        if (h == 0) p.out_scales[((size_t)(n0 / kMxGroup) * p.R + row) * 4 + (n0 / 32) % 4] = (uint8_t)byte;
    } else if constexpr (OUT == MOE_F32) {
        if (!live) return;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4_t *>(reinterpret_cast<float *>(p.out) + (size_t)row * p.N + n0 + 8 * q + 4 * h) =
                f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    } else {
        if (!live) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint16_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = OUT == MOE_BF16 ? to_bf16_rne(v[4 * q + i]) : __builtin_bit_cast(uint16_t, (_Float16)v[4 * q + i]);
            *reinterpret_cast<u32x2_t *>(reinterpret_cast<uint16_t *>(p.out) + (size_t)row * p.N + n0 + 8 * q + 4 * h) =
                u32x2_t{(uint32_t)b[0] | ((uint32_t)b[1] << 16), (uint32_t)b[2] | ((uint32_t)b[3] << 16)};
        }
    }
}

}  // namespace moe
