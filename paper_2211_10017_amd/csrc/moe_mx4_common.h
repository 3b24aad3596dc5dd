// The microscaled 4-bit format (OCP MX, e2m1 codes with an E8M0 scale per block of 32) on the device.
//
// A matrix of `rows` rows of K values, blocks of 32 along K:
//   codes  [rows, K/2] bytes, even k in the low nibble: a block is 16 contiguous bytes, which is what a lane feeds to
//          v_mfma_scale_f32_32x32x64_f8f6f4 as they are;
//   scales [ceil(K/128), rows, 4] bytes: byte b of group g is the scale of block 4 g + b.  A dword holds a row's four blocks of 128
//          values, and the dwords of 32 rows are one 128-byte line whatever K is (row-major scales of K = 2880 would be 90 bytes a row, no two rows
//          of them aligned alike).
// Scale byte s stands for 2^(s - 127), 255 for "not a number".
#pragma once

#include "moe_ffn_common.h"

namespace moe {

constexpr int kMxBlock = 32;
constexpr int kMxGroup = 128;                       // values whose four scales share a dword
__host__ __device__ inline int mx_groups(int K) { return K / kMxGroup + (K % kMxGroup != 0); }
__host__ __device__ inline size_t mx_code_bytes(size_t rows, int K) { return rows * (size_t)(K / 2); }
__host__ __device__ inline size_t mx_scale_bytes(size_t rows, int K) { return rows * 4 * (size_t)mx_groups(K); }

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Scale byte of a block whose largest magnitude has these bits: 2^(floor(log2 amax) - 2), the largest code being 6 = 1.5 * 2^2.  Subnormal amax
// (exponent field 0) and whatever is below the smallest scale take the smallest, infinities and NaN the byte for "not a number".
__device__ inline uint32_t mx_scale_byte(uint32_t amax_bits)
{
    const uint32_t field = amax_bits >> 23;                             // (the sign is not in it)
    return field == 255 ? 255 : field > 2 ? field - 2 : 0;
}

// The scale as the conversion instructions take it: an fp32 number of which they read the exponent field (field 0: 2^-127).
__device__ inline float mx_scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight values as codes in units of the scale, nearest, ties to the even code, saturating at 6.  Of a block that is not a number: zeros.
__device__ inline uint32_t mx_codes(const float (&v)[8], uint32_t byte)
{
    const float s = mx_scale_operand(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    return byte == 255 ? 0u : c;
}

__device__ inline float mx_scale_value(uint32_t byte)
{
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u);
}

// ---- one grouped product ---------------------------------------------------------------------------------------------------------
struct MxArgs {
    const uint8_t *a;         // codes [a_rows, K/2]
    const uint8_t *as;        // scales [ceil(K/128), a_rows, 4]
    const void *x;            // or null: rows [a_rows, K] that are not quantised yet, in x_dtype (16 bits); only where mx4_fuses_rows says so
    int x_dtype;
    int a_rows;
    const int32_t *a_src;     // [R] or null: row r is a[a_src[r] / a_div]
    int a_div;
    const int32_t *offsets;   // [E+1]
    const uint8_t *w;         // codes [E, N, K/2]
    const uint8_t *ws;        // scales [E, ceil(K/128), N, 4]
    const __half *bias;       // [E, N] or null
    void *out;                // [R, N] in out_dtype, or, with out_scales, codes [R, N/2]
    uint8_t *out_scales;      // [ceil(N/128), R, 4] or null
    int E, R, K, N;
    int most;                 // rows to choose a kernel for: R, or fewer if the caller knows
    int out_dtype, act;
};

int launch_mx4_gemm(const MxArgs &p, hipStream_t s);
bool mx4_fuses_rows(int most, int E, int N, int x_dtype);
int launch_mx4_tiled(const MxArgs &p, hipStream_t s);
int launch_mx4_quantize_rows(const void *x, int dtype, int R, int K, long stride, uint8_t *codes, uint8_t *scales, hipStream_t s);

}  // namespace moe
