// Grouped product of 4-bit rows and 4-bit experts in row tiles, for more rows per expert than one tile of the streaming kernel holds.
#include <type_traits>

#include "moe_mx4_epilogue.h"

namespace moe {

// Block: 2 x 2 wavefronts, a wavefront computes 32 TM rows by 32 TN channels.  Codes and scales of 128 values of K go from memory straight into a ring of
// NST stages in LDS: rows and channels alike are 64 bytes in it, 16-byte blocks at position block ^ ((row >> 2) & 3), so that sixteen rows' same block
// covers all banks, and one dword of scales.
template <int TM, int TN, int NST>
struct MxTile {
    static constexpr int BM = 64 * TM, BN = 64 * TN;
    static constexpr int kCodes = (BM + BN) * 64, kStage = kCodes + (BM + BN) * 4;
    static constexpr int NA = BM / 64, NB = BN / 64;                     // code loads per wavefront and stage (16 rows each)
    static constexpr int NC = ((BM + BN) / 64 + 3) / 4;                  // scale loads per wavefront and stage (64 rows each)
    static constexpr int L = NA + NB + NC;
    static constexpr int kLds = NST * kStage;
    static_assert(NST >= 3 && (NST - 3) * L < 64 && kLds <= 160 * 1024, "a stage in use, one arriving and one that is refilled");
};

template <int TM, int TN, int NST, int OUT>
__global__ __launch_bounds__(256, TM *TN > 8 ? 1 : 2) void mx4_tile_kernel(MxArgs p)
{
    using S = MxTile<TM, TN, NST>;
    constexpr int BM = S::BM, BN = S::BN, NA = S::NA, NB = S::NB, NC = S::NC, L = S::L;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave >> 1, wc = wave & 1;
    const int r = lane & 31, h = lane >> 5;
    const int K = p.K, N = p.N, G = mx_groups(K), blocks = K / kMxBlock;
    int e, col, row0, rows;
    if (!find_item(p.offsets, p.E, p.R, BM, (N + BN - 1) / BN, blockIdx.x, &e, &col, &row0, &rows)) return;
    e = __builtin_amdgcn_readfirstlane(e), col = __builtin_amdgcn_readfirstlane(col);
    row0 = __builtin_amdgcn_readfirstlane(row0), rows = __builtin_amdgcn_readfirstlane(rows);
    const int live = ((rows + 31) / 32 + 1) / 2;                        // row tiles of a wavefront that hold rows

    auto source = [&](int i) {                                          // row of `a` that row i of the block is (past the end: the last one)
        const int out_row = row0 + min(i, rows - 1);
        return p.a_src ? min(max(p.a_src[out_row] / p.a_div, 0), p.a_rows - 1) : out_row;
    };
    auto channel = [&](int i) { return min(col * BN + i, N - 1); };
    const int blk = (lane & 3) ^ ((lane >> 4) & 3);                     // the block of its row that this lane's loads bring
    const uint8_t *a_ptr[NA], *b_ptr[NB], *s_ptr[NC];
    long s_step[NC];
#pragma unroll
    for (int i = 0; i < NA; ++i) a_ptr[i] = p.a + (size_t)source((i * 4 + wave) * 16 + (lane >> 2)) * (K / 2) + blk * 16;
#pragma unroll
    for (int i = 0; i < NB; ++i) b_ptr[i] = p.w + ((size_t)e * N + channel((i * 4 + wave) * 16 + (lane >> 2))) * (K / 2) + blk * 16;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = (i * 4 + wave) % ((BM + BN) / 64);
        if (c < BM / 64) s_ptr[i] = p.as + (size_t)source(c * 64 + lane) * 4, s_step[i] = (long)p.a_rows * 4;
        else s_ptr[i] = p.ws + ((size_t)e * G * N + channel((c - BM / 64) * 64 + lane)) * 4, s_step[i] = (long)N * 4;
    }
    auto issue = [&](int s, int slot) {
        uint8_t *st = lds + slot * S::kStage;
        const int back = 4 * s + blk < blocks ? 0 : 32;                 // (the second half of the last group may not be there)
#pragma unroll
        for (int i = 0; i < NA; ++i) load_to_lds16(a_ptr[i] + s * 64 - back, reinterpret_cast<uint16_t *>(st + (i * 4 + wave) * 1024));
#pragma unroll
        for (int i = 0; i < NB; ++i) load_to_lds16(b_ptr[i] + s * 64 - back, reinterpret_cast<uint16_t *>(st + BM * 64 + (i * 4 + wave) * 1024));
#pragma unroll
        for (int i = 0; i < NC; ++i) load_to_lds4(s_ptr[i] + s * s_step[i], st + S::kCodes + (i * 4 + wave) % ((BM + BN) / 64) * 256);
    };

    float16_t acc[TM][TN] = {};
    auto run = [&](auto live_c) {
        constexpr int LIVE = decltype(live_c)::value;
        const int m0 = wr * LIVE * 32, n0 = wc * TN * 32;               // first row and channel of the wavefront
        u32x4_t a[2][LIVE], b[2][TN];
        uint32_t as[LIVE], bs[TN];
        auto read = [&](int slot, int j) {
            const uint8_t *st = lds + slot * S::kStage;
            const int at = r * 64 + (((2 * j + h) ^ ((r >> 2) & 3)) * 16);
#pragma unroll
            for (int n = 0; n < TN; ++n) b[j][n] = *reinterpret_cast<const u32x4_t *>(st + BM * 64 + (n0 + 32 * n) * 64 + at);
#pragma unroll
            for (int m = 0; m < LIVE; ++m) a[j][m] = *reinterpret_cast<const u32x4_t *>(st + (m0 + 32 * m) * 64 + at);
        };
        auto read_scales = [&](int slot) {
            const uint32_t *st = reinterpret_cast<const uint32_t *>(lds + slot * S::kStage + S::kCodes);
#pragma unroll
            for (int n = 0; n < TN; ++n) bs[n] = st[BM + n0 + 32 * n + r] >> (8 * h);
#pragma unroll
            for (int m = 0; m < LIVE; ++m) as[m] = st[m0 + 32 * m + r] >> (8 * h);
        };
        auto multiply = [&](auto j_c, const uint32_t (&as)[LIVE], const uint32_t (&bs)[TN]) {
            constexpr int J = decltype(j_c)::value;
#pragma unroll
            for (int m = 0; m < LIVE; ++m)
#pragma unroll
                for (int n = 0; n < TN; ++n)
                    acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        i32x8_t{(int)b[J][n][0], (int)b[J][n][1], (int)b[J][n][2], (int)b[J][n][3], 0, 0, 0, 0},
                        i32x8_t{(int)a[J][m][0], (int)a[J][m][1], (int)a[J][m][2], (int)a[J][m][3], 0, 0, 0, 0}, acc[m][n], 4, 4, 2 * J, (int)bs[n], 2 * J, (int)as[m]);
        };
        // Stage s + 1 has to be there when the wavefront is in the middle of stage s; the stages after it may still be on their way.  The barrier there
        // also says that everyone has read all of stage s - 1, whose place is refilled.
        for (int s = 0, slot = 0; s < G; ++s) {
            const int next = slot + 1 == NST ? 0 : slot + 1;
            if (s == 0) {
                wait_loads<0>();
                __syncthreads();
                read(slot, 0);
                read_scales(slot);
            }
            read(slot, 1);
            multiply(std::integral_constant<int, 0>{}, as, bs);
            uint32_t as1[LIVE], bs1[TN];
#pragma unroll
            for (int m = 0; m < LIVE; ++m) as1[m] = as[m];
#pragma unroll
            for (int n = 0; n < TN; ++n) bs1[n] = bs[n];
            if (s + 1 < G) {
                if (NST > 3 && s + 2 < G) wait_loads<(NST - 3) * L>();
                else wait_loads<0>();
                __syncthreads();
                read(next, 0);
                read_scales(next);
                if (s + NST - 1 < G) issue(s + NST - 1, slot == 0 ? NST - 1 : slot - 1);
            }
            if (4 * s + 2 < blocks) multiply(std::integral_constant<int, 1>{}, as1, bs1);
            slot = next;
        }
#pragma unroll
        for (int m = 0; m < LIVE; ++m)
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                const int i = m0 + 32 * m + r, c = col * BN + n0 + 32 * n;
                if (c < N) mx_store_tile<OUT>(p, acc[m][n], e, c, row0 + i, i < rows);
            }
    };
#pragma unroll
    for (int s = 0; s < NST - 1; ++s)
        if (s < G) issue(s, s);
    if (TM == 1 || live == 1) run(std::integral_constant<int, 1>{});
    else if (TM == 2 || live == 2) run(std::integral_constant<int, TM < 2 ? TM : 2>{});
    else if (live == 3) run(std::integral_constant<int, TM < 3 ? TM : 3>{});
    else run(std::integral_constant<int, TM>{});
}

template <int TM, int TN, int NST>
static int launch_tile(const MxArgs &p, hipStream_t s)
{
    using S = MxTile<TM, TN, NST>;
    const long slots = (long)p.R / S::BM + (p.E < p.R ? p.E : p.R);
    const long wgs = (slots * ((p.N + S::BN - 1) / S::BN) + kXcds - 1) / kXcds * kXcds;      // upper bound of the work items, whole rounds of XCDs
    if (wgs > 0xffffff) return fail(MOE_ERR_UNSUPPORTED, "moe_grouped_gemm_mx4: %ld workgroups exceed one launch", wgs);
    auto run = [&](auto out) {
        constexpr int OUT = decltype(out)::value;
        static std::atomic<uint64_t> raised;
        raise_lds_limit(reinterpret_cast<const void *>(&mx4_tile_kernel<TM, TN, NST, OUT>), S::kLds, raised);
        hipLaunchKernelGGL((mx4_tile_kernel<TM, TN, NST, OUT>), dim3((unsigned)wgs), dim3(256), S::kLds, s, p);
    };
    if (p.out_scales) run(std::integral_constant<int, -1>{});
    else if (p.out_dtype == MOE_F16) run(std::integral_constant<int, MOE_F16>{});
    else if (p.out_dtype == MOE_BF16) run(std::integral_constant<int, MOE_BF16>{});
    else run(std::integral_constant<int, MOE_F32>{});
    return check_launch("moe_grouped_gemm_mx4");
}

int launch_mx4_tiled(const MxArgs &p, int bm, hipStream_t s)
{
    if (bm == 64) return launch_tile<1, 4, 3>(p, s);
    if (bm == 128) return launch_tile<2, 4, 3>(p, s);
    return launch_tile<4, 4, 4>(p, s);
}

}  // namespace moe
