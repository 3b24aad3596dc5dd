// Grouped product of 4-bit rows and 4-bit experts for few rows per expert: a launch that streams weights.
#include <type_traits>

#include "moe_mx4_epilogue.h"

namespace moe {

// Block: WAVES wavefronts, one item of up to 32 rows of an expert by NS slabs of 32 channels; the wavefronts split K, 256 values (a line of a channel's
// codes) at a time, CPW of them each per pass, and their sums meet in LDS, added in the order of the wavefronts.  Weights go from memory into the
// wavefront's own part of LDS, eight channels' whole lines per load: requested first, before the block knows its rows, so that the chain of index and rows
// runs under them.  (Weights straight into registers, a channel's sixteen bytes per lane, touch 64 places per load: 29 us instead of 16.7 for 70 MB.)
// Rows' codes, of which there are few and which come from L2, and scales go into registers.
//
// Of 256 values lane (r, h) takes blocks 4 h .. 4 h + 3 of its channel (or row), and step j multiplies block 4 h + j of both operands: any pairing of
// blocks with steps will do as long as it is the same on both sides, and with this one the scales of a lane's four steps are one dword.
//
// XDT (MOE_F16 | MOE_BF16, or -1: codes): rows that are not quantised yet.  As a lane's operand is a whole block of its row, it quantises what it multiplies
// without a word to any other, which saves a launch where there are few blocks to repeat it (mx4_fuses_rows).
// A block of 32 16-bit values as codes, and its scale byte; the same bits as mx4_quantize_rows_kernel.
template <int XDT>
__device__ inline u32x4_t mx_quantize_block(const u32x4_t (&raw)[4], uint32_t &byte)
{
    typedef unsigned short us2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
    // (by value: the compiler's bit_cast of a vector's element is that of its first one)
    auto pair = [](uint32_t v) { return __builtin_bit_cast(bf2_t, v); };
    us2_t m = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2_t, raw[i >> 2][i & 3] & 0x7fff7fffu));
    const uint16_t top = m[0] > m[1] ? m[0] : m[1];
    byte = mx_scale_byte(XDT == MOE_BF16 ? (uint32_t)top << 16 : __float_as_uint((float)__builtin_bit_cast(_Float16, top)));
    const float s = mx_scale_operand(byte);
    u32x4_t c;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t d = 0;
        if constexpr (XDT == MOE_BF16) {
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(d, pair(raw[q][0]), s, 0);
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(d, pair(raw[q][1]), s, 1);
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(d, pair(raw[q][2]), s, 2);
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(d, pair(raw[q][3]), s, 3);
        } else {
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(d, bits_h2(raw[q][0]), s, 0);
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(d, bits_h2(raw[q][1]), s, 1);
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(d, bits_h2(raw[q][2]), s, 2);
            d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(d, bits_h2(raw[q][3]), s, 3);
        }
        c[q] = byte == 255 ? 0u : d;
    }
    return c;
}

template <int WAVES, int NS, int CPW>
struct MxStream {
    static constexpr int kWave = NS * CPW * 4096;
    static constexpr int kLds = WAVES * kWave;          // (the partial sums, 4 KB per wavefront and slab, fit as well)
};

template <int WAVES, int NS, int CPW, int OUT, int XDT>
__global__ __launch_bounds__(64 * WAVES) void mx4_stream_kernel(MxArgs p)
{
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5;
    const int K = p.K, N = p.N, G = mx_groups(K), blocks = K / kMxBlock, chunks = (blocks + 7) / 8;
    int e, col, row0, rows;
    if (!find_item(p.offsets, p.E, p.R, 32, (N + 32 * NS - 1) / (32 * NS), blockIdx.x, &e, &col, &row0, &rows)) return;
    e = __builtin_amdgcn_readfirstlane(e), col = __builtin_amdgcn_readfirstlane(col);
    row0 = __builtin_amdgcn_readfirstlane(row0), rows = __builtin_amdgcn_readfirstlane(rows);
    const int n0 = col * 32 * NS;
    const uint8_t *w = p.w + (size_t)e * N * (K / 2);
    const uint32_t *ws = reinterpret_cast<const uint32_t *>(p.ws) + (size_t)e * G * N;
    uint8_t *mine = lds + wave * MxStream<WAVES, NS, CPW>::kWave;

    // (channels past N: the last slab again, not stored; chunks past K: whatever LDS holds, times rows of zeros)
    auto slab = [&](int s) { return min(n0 + 32 * s, N - 32); };
    auto request = [&](int pass) {
#pragma unroll
        for (int i = 0; i < CPW; ++i) {
            const int c = (pass * CPW + i) * WAVES + wave;
            if (c >= chunks) break;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int row = 8 * t + (lane >> 3), b = min(8 * c + ((lane & 7) ^ ((row >> 1) & 7)), blocks - 1);
                    load_to_lds16<true>(w + (size_t)(slab(s) + row) * (K / 2) + (size_t)b * 16, reinterpret_cast<uint16_t *>(mine + ((i * NS + s) * 4 + t) * 1024));
                }
        }
    };
    request(0);
    const int out_row = row0 + min(r, rows - 1);             // (lanes past the rows repeat the last one)
    const int a_row = p.a_src ? min(max(p.a_src[out_row] / p.a_div, 0), p.a_rows - 1) : out_row;
    const uint8_t *a = XDT < 0 ? p.a + (size_t)a_row * (K / 2) : reinterpret_cast<const uint8_t *>(p.x) + (size_t)a_row * K * 2;
    const uint32_t *as = reinterpret_cast<const uint32_t *>(p.as) + a_row;

    float16_t acc[NS] = {};
    for (int pass = 0; pass * CPW * WAVES < chunks; ++pass) {
        if (pass) request(pass);
        u32x4_t aq[CPW][4];
        uint32_t asc[CPW], wsc[CPW][NS];
#pragma unroll
        for (int i = 0; i < CPW; ++i) {
            const int b0 = 8 * ((pass * CPW + i) * WAVES + wave) + 4 * h;          // this lane's blocks, and their group of scales
            const int g = min(b0 / 4, G - 1);
            // scales of blocks that are not there may hold anything; the rows' codes are zero there
            const uint32_t mask = b0 + 4 <= blocks ? 0xffffffffu : b0 < blocks ? (1u << (8 * (blocks - b0))) - 1 : 0;
            if constexpr (XDT < 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    aq[i][j] = u32x4_t{};
                    if (b0 + j < blocks) aq[i][j] = *reinterpret_cast<const u32x4_t *>(a + (size_t)(b0 + j) * 16);
                }
                asc[i] = as[(size_t)g * p.a_rows] & mask;
            } else {
                u32x4_t raw[4][4] = {};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (b0 + j < blocks)
#pragma unroll
                        for (int q = 0; q < 4; ++q) raw[j][q] = *reinterpret_cast<const u32x4_t *>(a + (size_t)(b0 + j) * 64 + q * 16);
                asc[i] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t byte;
                    aq[i][j] = mx_quantize_block<XDT>(raw[j], byte);
                    asc[i] |= byte << (8 * j);
                }
            }
#pragma unroll
            for (int s = 0; s < NS; ++s) wsc[i][s] = ws[(size_t)g * N + slab(s) + r] & mask;
        }
        wait_loads<0>();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < CPW; ++i)
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                u32x4_t wq[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    wq[j] = *reinterpret_cast<const u32x4_t *>(mine + (i * NS + s) * 4096 + r * 128 + (((4 * h + j) ^ ((r >> 1) & 7)) * 16));
                auto step = [&](auto j_c) {
                    constexpr int J = decltype(j_c)::value;
                    acc[s] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        i32x8_t{(int)wq[J][0], (int)wq[J][1], (int)wq[J][2], (int)wq[J][3], 0, 0, 0, 0},
                        i32x8_t{(int)aq[i][J][0], (int)aq[i][J][1], (int)aq[i][J][2], (int)aq[i][J][3], 0, 0, 0, 0}, acc[s], 4, 4, J, (int)wsc[i][s], J, (int)asc[i]);
                };
                step(std::integral_constant<int, 0>{});
                step(std::integral_constant<int, 1>{});
                step(std::integral_constant<int, 2>{});
                step(std::integral_constant<int, 3>{});
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the next pass's weights take the place of these)
    }
    __syncthreads();
    f32x4_t *part = reinterpret_cast<f32x4_t *>(lds);               // [wavefront][slab][q][lane]
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            part[((wave * NS + s) * 4 + q) * 64 + lane] = f32x4_t{acc[s][4 * q], acc[s][4 * q + 1], acc[s][4 * q + 2], acc[s][4 * q + 3]};
    __syncthreads();
    if (wave >= NS || n0 + 32 * wave >= N) return;
    float16_t sum;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f32x4_t v = part[(wave * 4 + q) * 64 + lane];
#pragma unroll
        for (int t = 1; t < WAVES; ++t) v += part[((t * NS + wave) * 4 + q) * 64 + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[4 * q + i] = v[i];
    }
    mx_store_tile<OUT>(p, sum, e, n0 + 32 * wave, row0 + r, r < rows);
}

template <int WAVES, int NS, int CPW>
static int launch_stream(const MxArgs &p, hipStream_t s)
{
    using S = MxStream<WAVES, NS, CPW>;
    const long slots = (long)p.R / 32 + (p.E < p.R ? p.E : p.R);
    const long wgs = (slots * ((p.N + 32 * NS - 1) / (32 * NS)) + kXcds - 1) / kXcds * kXcds;      // upper bound of the work items, whole rounds of XCDs
    if (wgs * WAVES > 0x3ffffff) return fail(MOE_ERR_UNSUPPORTED, "moe_grouped_gemm_mx4: %ld workgroups exceed one launch", wgs);
    auto run = [&](auto out, auto x) {
        constexpr int OUT = decltype(out)::value, XDT = decltype(x)::value;
        hipLaunchKernelGGL((mx4_stream_kernel<WAVES, NS, CPW, OUT, XDT>), dim3((unsigned)wgs), dim3(64 * WAVES), S::kLds, s, p);
    };
    static_assert(S::kLds <= 64 * 1024, "what a launch may ask for without more");
    using std::integral_constant;
    constexpr integral_constant<int, -1> codes{};
    if constexpr (NS == 1) {                             // (mx4_fuses_rows: of few blocks, which are those of one slab)
        if (p.x && p.x_dtype == MOE_F16) return run(codes, integral_constant<int, MOE_F16>{}), check_launch("moe_grouped_ffn_mx4");
        if (p.x) return run(codes, integral_constant<int, MOE_BF16>{}), check_launch("moe_grouped_ffn_mx4");
    } else if (p.x) return fail(MOE_ERR_UNSUPPORTED, "moe_grouped_ffn_mx4: rows that are not quantised, for %d slabs", NS);
    if (p.out_scales) run(codes, codes);
    else if (p.out_dtype == MOE_F16) run(integral_constant<int, MOE_F16>{}, codes);
    else if (p.out_dtype == MOE_BF16) run(integral_constant<int, MOE_BF16>{}, codes);
    else run(integral_constant<int, MOE_F32>{}, codes);
    return check_launch("moe_grouped_gemm_mx4");
}

// Wavefronts, slabs and lines per wavefront of a block (kernel times in us, 4 KB of LDS for each of the three; what counts is how many bytes a compute unit has in
// flight, so small blocks, and how often a block's chain of index and rows is paid for, so not too small ones):
//  - few blocks: one slab, and K in as few rounds as wavefronts allow (16 tokens, two of 32 experts, fc2 of 4096 x 1024: eight wavefronts 10.3, four with two slabs 11.7);
//  - K up to 1024: four wavefronts, one slab (64 tokens, two of 32 experts, 1024 x 4096: 16.7, two slabs 16.8, four 18.1; 40 tokens, one each, 12.4 / 13.2 / 13.7);
//  - K up to 4096 and many blocks: two wavefronts with two slabs and two lines (64 tokens, two of 32 experts, 2048 x 8192: 48.9 = 5.7 TB/s, eight wavefronts 59.5;
//    of 64 experts of 4096 x 16384 281 and 285 to 329); fewer: four wavefronts, two slabs (64 tokens, 4096 x 1024: 13.4, eight wavefronts 14.2);
//  - longer K: eight wavefronts, two slabs (8192 x 2048: 46.6 = 6.0 TB/s, two wavefronts 58.1; 16384 x 4096 286 and 291).
// Row tiles from 25 rows per expert on.  One bound on the mean for all products, which is where an FFN's two together are about as fast either way (us, fc1 + fc2, streaming / tiles,
// two of 32 experts): of 1024 x 4096 16 rows 20.4 + 16.9 / 18.7 + 20.1, 24 rows 21.3 + 20.7 / 19.1 + 19.8, 32 rows 27.7 + 22.4 / 19.7 + 20.5; of 2048 x 8192 24 rows 65 + 59 / 64 + 69.
// What it gives away: 1 to 2 us of a product with short K at 16 to 24 rows, which tiles would win, and an expert with much of an uneven batch, which is streamed in items of
// 32 rows that each read its weights.
static bool streams(int most, int E) { return ((long)most + E - 1) / E <= 24; }

int launch_mx4_gemm(const MxArgs &p, hipStream_t s)
{
    if (!streams(p.most, p.E)) return launch_mx4_tiled(p, s);
    const double blocks = decode_active_experts(p.most, p.E) * (p.N / 64);
    if (p.K <= 1024) return launch_stream<4, 1, 1>(p, s);
    if (blocks < 450) return launch_stream<8, 1, 1>(p, s);
    if (p.K > 4096) return launch_stream<8, 2, 1>(p, s);
    return blocks >= 2048 ? launch_stream<2, 2, 2>(p, s) : launch_stream<4, 2, 1>(p, s);
}

// Whether fc1 quantises its rows for itself: every block does so for the rows of its item, so only where there are few blocks.  An FFN of two experts a token, us, by itself / after the
// quantiser: 32 experts of 1024 x 4096, fp16, 252 blocks 10.8 / 12.0, 488 12.0 / 12.7, 919 15.5 / 14.9; bf16 10.5 / 11.8, 12.5 / 13.1, 16.0 / 15.4; 16 of 704 x 2880, 581 blocks 12.6 / 12.9, 927
// 13.9 / 13.7; 32 of 512 x 2048, 816 blocks 11.9 / 11.7.  Longer rows want fewer blocks, which the bound leaves aside: 4096 x 1024, 230 blocks 14.5 / 14.9, 408 20.9 / 18.9; 2048 x 8192, 448 17.0 / 16.4.
bool mx4_fuses_rows(int most, int E, int N, int x_dtype)
{
    return x_dtype != MOE_F32 && streams(most, E) && decode_active_experts(most, E) * (N / 32) <= 512;
}

}  // namespace moe
