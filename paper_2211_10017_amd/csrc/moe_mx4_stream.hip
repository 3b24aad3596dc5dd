// Grouped product of 4-bit rows and 4-bit experts for few rows per expert.
#include "moe_mx4_epilogue.h"

namespace moe {

// Block: four wavefronts, one item of up to 32 rows of an expert by 32 channels; the wavefronts take every fourth 256 values of K and their sums meet
// in LDS, added in the order of the wavefronts.  Codes go from memory to registers as the matrix instruction wants them: of 256 values lane (r, h)
// takes the 64 bytes that are blocks 4 h .. 4 h + 3 of its channel (or row), so the two lanes of a channel read a whole line, and step j multiplies
// block 4 h + j of both operands: any pairing of blocks with steps will do as long as it is the same on both sides, and with this one
// the scales of a lane's four steps are one dword.
constexpr int kStreamWaves = 4;

template <int OUT>
__global__ __launch_bounds__(256) void mx4_stream_kernel(MxArgs p)
{
    __shared__ f32x4_t part[kStreamWaves][4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5;
    const int K = p.K, N = p.N, G = mx_groups(K), blocks = K / kMxBlock;
    int e, col, row0, rows;
    if (!find_item(p.offsets, p.E, p.R, 32, N / 32, blockIdx.x, &e, &col, &row0, &rows)) return;
    e = __builtin_amdgcn_readfirstlane(e), col = __builtin_amdgcn_readfirstlane(col);
    row0 = __builtin_amdgcn_readfirstlane(row0), rows = __builtin_amdgcn_readfirstlane(rows);
    const int n = col * 32 + r, out_row = row0 + min(r, rows - 1);             // (lanes past the rows repeat the last one)
    const int a_row = p.a_src ? min(max(p.a_src[out_row] / p.a_div, 0), p.a_rows - 1) : out_row;
    const uint8_t *w = p.w + ((size_t)e * N + n) * (K / 2), *a = p.a + (size_t)a_row * (K / 2);
    const uint32_t *ws = reinterpret_cast<const uint32_t *>(p.ws) + (size_t)e * G * N + n;
    const uint32_t *as = reinterpret_cast<const uint32_t *>(p.as) + a_row;

    float16_t acc = {};
    for (int c = wave; c * 256 < K; c += kStreamWaves) {
        const int b0 = 8 * c + 4 * h, g = 2 * c + h;                           // this lane's blocks and their group of scales
        u32x4_t wq[4] = {}, aq[4] = {};
        uint32_t wsc = 0, asc = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (b0 + j < blocks) {
                wq[j] = *reinterpret_cast<const u32x4_t *>(w + (size_t)(b0 + j) * 16);
                aq[j] = *reinterpret_cast<const u32x4_t *>(a + (size_t)(b0 + j) * 16);
            }
        if (b0 < blocks) wsc = ws[(size_t)g * N], asc = as[(size_t)g * p.a_rows];
        if (b0 + 4 > blocks) {                                                 // scales of blocks that are not there may hold anything
            const uint32_t mask = b0 < blocks ? (1u << (8 * (blocks - b0))) - 1 : 0;
            wsc &= mask, asc &= mask;
        }
#define MX_STEP(J)                                                                                                                                     \
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(i32x8_t{(int)wq[J][0], (int)wq[J][1], (int)wq[J][2], (int)wq[J][3], 0, 0, 0, 0},            \
                                                          i32x8_t{(int)aq[J][0], (int)aq[J][1], (int)aq[J][2], (int)aq[J][3], 0, 0, 0, 0}, acc, 4, 4, \
                                                          J, (int)wsc, J, (int)asc)
        MX_STEP(0);
        MX_STEP(1);
        MX_STEP(2);
        MX_STEP(3);
#undef MX_STEP
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) part[wave][q][lane] = f32x4_t{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f32x4_t s = part[0][q][lane];
#pragma unroll
        for (int t = 1; t < kStreamWaves; ++t) s += part[t][q][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[4 * q + i] = s[i];
    }
    mx_store_tile<OUT>(p, acc, e, col * 32, row0 + r, r < rows);
}

int launch_mx4_gemm(const MxArgs &p, hipStream_t s)
{
    const int mean = (p.R + p.E - 1) / p.E;
    if (mean > 24) return launch_mx4_tiled(p, mean <= 64 ? 64 : mean <= 128 ? 128 : 256, s);
    const long slots = (long)p.R / 32 + (p.E < p.R ? p.E : p.R);
    const long wgs = (slots * (p.N / 32) + kXcds - 1) / kXcds * kXcds;         // upper bound of the work items, whole rounds of XCDs
    if (wgs > 0xffffff) return fail(MOE_ERR_UNSUPPORTED, "moe_grouped_gemm_mx4: %ld workgroups exceed one launch", wgs);
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, s, p); };
    if (p.out_scales) run(&mx4_stream_kernel<-1>);
    else if (p.out_dtype == MOE_F16) run(&mx4_stream_kernel<MOE_F16>);
    else if (p.out_dtype == MOE_BF16) run(&mx4_stream_kernel<MOE_BF16>);
    else run(&mx4_stream_kernel<MOE_F32>);
    return check_launch("moe_grouped_gemm_mx4");
}

}  // namespace moe
