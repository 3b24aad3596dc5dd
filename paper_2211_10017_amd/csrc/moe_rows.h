// Rows of 16- and 32-bit floats: a thread's neighbouring channels as fp32 numbers, and back with one rounding.
#pragma once

#include <type_traits>

#include "moe_ffn_common.h"

namespace moe {

constexpr int size_of(int dtype) { return dtype == MOE_F32 ? 4 : 2; }

// V neighbouring values as they lie in memory: 8, 16 or 32 bytes.
template <int DT, int V>
struct Raw {
    static constexpr int WORDS = V * size_of(DT) / 4;
    static_assert(WORDS == 2 || WORDS % 4 == 0, "loads of eight or sixteen bytes");
    uint32_t w[WORDS];

    __device__ inline void load(const void *base, size_t at)                // at: the first value's index, a multiple of V
    {
        const char *p = reinterpret_cast<const char *>(base) + at * size_of(DT);
        if constexpr (WORDS == 2) {
            const uint2 q = *reinterpret_cast<const uint2 *>(p);
            w[0] = q.x, w[1] = q.y;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
                const uint4 q = *reinterpret_cast<const uint4 *>(p + 4 * i);
                w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
            }
        }
    }
    __device__ inline void store(void *base, size_t at) const
    {
        char *p = reinterpret_cast<char *>(base) + at * size_of(DT);
        if constexpr (WORDS == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) *reinterpret_cast<uint4 *>(p + 4 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        }
    }
    __device__ inline void clear()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ inline float get(int i) const
    {
        if (DT == MOE_F32) return __uint_as_float(w[i % WORDS]);
        if (DT == MOE_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        return (float)__builtin_bit_cast(half2_t, w[i / 2])[i & 1];
    }
    __device__ inline void set(const float (&v)[V])
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if (DT == MOE_F32) w[i] = __float_as_uint(v[i % V]);
            else if (DT == MOE_BF16) w[i] = to_bf16_rne(v[2 * i % V]) | (uint32_t)to_bf16_rne(v[(2 * i + 1) % V]) << 16;
            else w[i] = h2_bits(half2_t{(_Float16)v[2 * i % V], (_Float16)v[(2 * i + 1) % V]});
        }
    }
};

template <int DT>
__device__ inline float load_one(const void *base, size_t at)
{
    if (DT == MOE_F32) return reinterpret_cast<const float *>(base)[at];
    const uint16_t b = reinterpret_cast<const uint16_t *>(base)[at];
    return DT == MOE_BF16 ? __uint_as_float((uint32_t)b << 16) : (float)__builtin_bit_cast(_Float16, b);
}

template <int DT>
__device__ inline void store_one(void *base, size_t at, float v)
{
    if (DT == MOE_F32) reinterpret_cast<float *>(base)[at] = v;
    else reinterpret_cast<uint16_t *>(base)[at] = DT == MOE_BF16 ? to_bf16_rne(v) : __builtin_bit_cast(uint16_t, (_Float16)v);
}

// f(integral_constant of the element type) for a type known on the host.
template <class F>
inline int with_dtype(int dtype, F &&f)
{
    if (dtype == MOE_F16) return f(std::integral_constant<int, MOE_F16>{});
    if (dtype == MOE_BF16) return f(std::integral_constant<int, MOE_BF16>{});
    return f(std::integral_constant<int, MOE_F32>{});
}
inline bool known_dtype(int dtype) { return dtype == MOE_F16 || dtype == MOE_BF16 || dtype == MOE_F32; }

__device__ inline float wave_sum(float v)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

}  // namespace moe
