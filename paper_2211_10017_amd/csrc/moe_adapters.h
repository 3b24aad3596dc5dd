// What the adapters' kernels share: arguments, and how coefficients go into 16-bit products.
#pragma once

#include "moe_rows.h"

namespace moe {

constexpr int kAdapterMostRank = 128, kAdapterMostAdapters = 4096;
constexpr int kAdapterMostRows = 1 << 30;           // a row's number and the steps that are requested ahead of it (two of 32 rows, or the next part's) stay below 2^31
constexpr int kAdapterRowsWithoutV = 512;           // more rows take two launches, between which the coefficients are in memory

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));

// Where row r of the sorted order is found: in rows of tokens (source / div), of assignments (source), or in place.
struct RowMap {
    const int32_t *source;      // perm_src or null
    int div;                    // k for tokens, 1 for assignments
    int rows;                   // of the buffer
    int64_t stride;

    // Several rows at once: their loads are requested together.
    template <int N>
    __device__ inline void find(int (&r)[N]) const
    {
        if (!source) return;
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = source[r[i]];
        if (div == 2) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] >>= 1;
        } else if (div != 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] /= div;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = min(max(r[i], 0), rows - 1);
    }
};

// f(integral_constant 0), ... f(integral_constant N - 1)
template <int N, class F, int I = 0>
__device__ inline void unrolled(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<N, F &, I + 1>(f);
    }
}

// Requests stand ahead of what is done while they are under way: left to itself the compiler moves them behind it.
__device__ inline void requested() { __builtin_amdgcn_sched_barrier(0); }

// coef[r] = A[e] x[r] (for phase two times scale[e]), out[r] = y[r] + coef[r] B[e]
struct AdapterArgs {
    const int32_t *offsets;     // [E + 1]
    const float *scale;         // [E] or null
    int R, E, K, N, rank;
    const void *x, *a, *b;
    RowMap x_map;
    const void *y;              // or null; may be out
    int64_t y_stride;
    void *out;
    RowMap out_map;             // of y as well, but for the stride
    float *coef;                // [R, rank], or null (one launch does without)
    int coef_scaled;            // coef holds scale * (A x)
    int ncol;                   // slices of N, each a block's
    int width;                  // channels of a slice, a multiple of 64
    int items;                  // blocks for rows of adapters; those behind them copy the others
    int share;                  // rows of a block, about
};

// out[e][j] = scale sum_r coef[r][j] rows[r]
struct OuterJob {
    const void *rows;
    RowMap map;
    const float *coef;          // [R, rank]
    const float *scale;         // [E] or null
    void *out;                  // [E, rank, C] or null: no such job
    int C, ncol;                // ncol: slices of 64 channels
    int chunk;                  // rows of a block, a multiple of 32
    float *part;                // [slots, rank, C]: sums of adapters with more than one chunk
    int slots;                  // enough for every partition of the R rows
};
struct OuterArgs {
    const int32_t *offsets;
    int R, E, rank, out_dtype;
    OuterJob job[2];
    int first, items;           // blocks of job 0, and of both (the grid is rounded up; a job without `out` has none)
    int turns;                  // parts of the rank
    int join;                   // adapters that can have more than one chunk
};

// Forward: x in the adapters' type.  Backward: `x` is dy, of any type, and out is dx, in the adapters'.
int launch_adapter_forward_f16(const AdapterArgs &p, int out_dtype, hipStream_t s, const char *what);
int launch_adapter_forward_bf16(const AdapterArgs &p, int out_dtype, hipStream_t s, const char *what);
int launch_adapter_backward_f16(const AdapterArgs &p, int x_dtype, hipStream_t s, const char *what);
int launch_adapter_backward_bf16(const AdapterArgs &p, int x_dtype, hipStream_t s, const char *what);
int launch_adapter_outer(const OuterArgs &p, int dtype0, int dtype1, hipStream_t s, const char *what);

template <int DT>
__device__ inline float4_t product16(u32x4_t a, u32x4_t b, float4_t c)          // 16 x 16 x 32
{
    if constexpr (DT == MOE_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));

template <int DT>
__device__ inline float4_t product16(u32x2_t a, u32x2_t b, float4_t c)          // 16 x 16 x 16
{
    if constexpr (DT == MOE_BF16) return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4_t, a), __builtin_bit_cast(short4_t, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(half4_t, a), __builtin_bit_cast(half4_t, b), c, 0, 0, 0);
}

// A coefficient as 16-bit terms, each the nearest to what those before it leave: two are off by at most 2^-16 of it in bf16 and 2^-22 in fp16, where one alone would be off by
// 2^-8 and 2^-11, as much as a 16-bit result may be altogether; in bf16 a third (2^-24) where the result is fp32.  (fp16: of numbers that a power of two has brought into range.)
template <int DT>
struct Split {
    uint16_t hi, lo, rest;
    __device__ inline explicit Split(float c)
    {
        hi = take(c);
        c = __builtin_isfinite(c) ? c : 0.0f;                   // (an infinity leaves none, nor does a number that becomes one in bf16; what finite numbers leave is finite)
        lo = take(c), rest = DT == MOE_BF16 ? take(c) : 0;
    }
    __device__ static inline uint16_t take(float &c)
    {
        using T = std::conditional_t<DT == MOE_BF16, __bf16, _Float16>;
        const T h = (T)c;
        c -= (float)h;
        return __builtin_bit_cast(uint16_t, h);
    }
};

// The power of two that numbers of up to `most` are divided by before they are split in fp16: the largest then lies in [2^14, 2^15) (infinities stay infinities).
__device__ inline int split_exponent(float most)
{
    const int e = (int)(__float_as_uint(most) >> 23) - 127 - 14;
    return min(max(e, -100), 100);
}
__device__ inline float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }       // -126 <= e <= 127

// Four columns of four or eight rows, a row's four as two words, become the columns: column t's values as words.
template <int ROWS, class Operand>
__device__ inline void transpose_columns(const uint2 (&row)[ROWS], Operand (&col)[4])
{
#pragma unroll
    for (int i = 0; i < ROWS / 2; ++i) {
        col[0][i] = __builtin_amdgcn_perm(row[2 * i + 1].x, row[2 * i].x, 0x05040100u);
        col[1][i] = __builtin_amdgcn_perm(row[2 * i + 1].x, row[2 * i].x, 0x07060302u);
        col[2][i] = __builtin_amdgcn_perm(row[2 * i + 1].y, row[2 * i].y, 0x05040100u);
        col[3][i] = __builtin_amdgcn_perm(row[2 * i + 1].y, row[2 * i].y, 0x07060302u);
    }
}

}  // namespace moe
