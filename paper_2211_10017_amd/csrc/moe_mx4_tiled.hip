// Grouped product of 4-bit rows and 4-bit experts in row tiles, for more rows per expert than one tile of the streaming kernel holds.
#include <type_traits>

#include "moe_mx4_epilogue.h"

namespace moe {

// Block: WR x WC wavefronts, a wavefront computes 32 TM rows by 32 TN channels.  Codes and scales of 128 values of K go from memory straight into a ring of
// NST stages in LDS: rows and channels alike are 64 bytes in it, 16-byte blocks at position block ^ ((row >> 2) & 3), so that sixteen rows' same block
// covers all banks, and one dword of scales.
template <int WR, int WC, int TM, int TN, int NST>
struct MxTile {
    static constexpr int W = WR * WC, BM = 32 * TM * WR, BN = 32 * TN * WC;
    static constexpr int kCodes = (BM + BN) * 64, kStage = kCodes + (BM + BN) * 4;
    static constexpr int NA = BM / 16 / W, NB = BN / 16 / W;             // code loads per wavefront and stage (16 rows each)
    static constexpr int NCA = (BM / 64 + W - 1) / W, NCB = (BN / 64 + W - 1) / W;      // scale loads (64 rows each)
    static constexpr int LA = NA + NCA, L = LA + NB + NCB;
    static constexpr int kLds = NST * kStage;
    static constexpr int kPerCu = 160 * 1024 / kLds < 1 ? 1 : 160 * 1024 / kLds;
    static_assert(BM % (16 * W) == 0 && BN % (16 * W) == 0, "loads are dealt evenly");
    static_assert(NST >= 2 && NST <= 3 && (NST - 1) * L < 64 && kLds <= 160 * 1024, "a stage in use and one or more on their way");
};

template <int WR, int WC, int TM, int TN, int NST, int OUT>
__global__ __launch_bounds__(64 * WR * WC, TM *TN > 8 ? 1 : 2) void mx4_tile_kernel(MxArgs p)
{
    using S = MxTile<WR, WC, TM, TN, NST>;
    constexpr int W = S::W, BM = S::BM, BN = S::BN, NA = S::NA, NB = S::NB, NCA = S::NCA, NCB = S::NCB, LA = S::LA, L = S::L;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
    const int r = lane & 31, h = lane >> 5;
    const int K = p.K, N = p.N, G = mx_groups(K), blocks = K / kMxBlock;
    int e, col, row0, rows;
    if (!find_item(p.offsets, p.E, p.R, BM, (N + BN - 1) / BN, blockIdx.x, &e, &col, &row0, &rows)) return;
    e = __builtin_amdgcn_readfirstlane(e), col = __builtin_amdgcn_readfirstlane(col);
    row0 = __builtin_amdgcn_readfirstlane(row0), rows = __builtin_amdgcn_readfirstlane(rows);
    const int live = ((rows + 31) / 32 + WR - 1) / WR;                  // row tiles of a wavefront that hold rows

    auto source = [&](int i) {                                          // row of `a` that row i of the block is (past the end: the last one)
        const int out_row = row0 + min(i, rows - 1);
        return p.a_src ? min(max(p.a_src[out_row] / p.a_div, 0), p.a_rows - 1) : out_row;
    };
    const int blk = (lane & 3) ^ ((lane >> 4) & 3);                     // the block of its row that this lane's loads bring
    // Weights and scales: a base of the wavefront's and an offset per lane, so that going on to the next stage costs no vector instruction; rows, which may lie
    // further apart than 32 bits reach, as pointers.
    const int c0 = col * BN;
    auto channel = [&](int i) { return (uint32_t)(min(c0 + i, N - 1) - c0); };
    const uint8_t *w = p.w + ((size_t)e * N + c0) * (K / 2), *ws = p.ws + ((size_t)e * G * N + c0) * 4, *as = p.as;
    uint32_t b_off[NB], bs_off[NCB], as_off[NCA];
    const uint8_t *a_ptr[NA];
    // (the second half of the last group may not be there: its lanes bring the first again)
    auto back = [&](int s) { return 4 * s + blk < blocks ? 0 : 32; };
    auto issue_weights = [&](int s, uint8_t *st) {                      // a stage's loads, to st in LDS
        const int b = back(s);
#pragma unroll
        for (int i = 0; i < NB; ++i) load_to_lds16_at(w, b_off[i] - b, st + BM * 64 + (i * W + wave) * 1024);
#pragma unroll
        for (int i = 0; i < NCB; ++i) load_to_lds4_at(ws, bs_off[i], st + S::kCodes + BM * 4 + (i * W + wave) % (BN / 64) * 256);
        w += 64, ws += (size_t)N * 4;
    };
    auto issue_rows = [&](int s, uint8_t *st) {
        const int b = back(s);
#pragma unroll
        for (int i = 0; i < NA; ++i) load_to_lds16(a_ptr[i] - b, reinterpret_cast<uint16_t *>(st + (i * W + wave) * 1024)), a_ptr[i] += 64;
#pragma unroll
        for (int i = 0; i < NCA; ++i) load_to_lds4_at(as, as_off[i], st + S::kCodes + (i * W + wave) % (BM / 64) * 256);
        as += (size_t)p.a_rows * 4;
    };
    // The first stages' weights are requested before the rows are known, so that the chain of index and rows runs under them.
    // (A lane steps back only from blocks 2 and 3, so its offset stays positive.)
#pragma unroll
    for (int i = 0; i < NB; ++i) b_off[i] = channel((i * W + wave) * 16 + (lane >> 2)) * (uint32_t)(K / 2) + blk * 16;
#pragma unroll
    for (int i = 0; i < NCB; ++i) bs_off[i] = channel((i * W + wave) % (BN / 64) * 64 + lane) * 4;
#pragma unroll
    for (int s = 0; s < NST; ++s)
        if (s < G) issue_weights(s, lds + s * S::kStage);
#pragma unroll
    for (int i = 0; i < NA; ++i) a_ptr[i] = p.a + (size_t)source((i * W + wave) * 16 + (lane >> 2)) * (K / 2) + blk * 16;
#pragma unroll
    for (int i = 0; i < NCA; ++i) as_off[i] = (uint32_t)source((i * W + wave) % (BM / 64) * 64 + lane) * 4;
#pragma unroll
    for (int s = 0; s < NST; ++s)
        if (s < G) issue_rows(s, lds + s * S::kStage);
    auto run = [&](auto live_c) {
        constexpr int LIVE = decltype(live_c)::value;
        float16_t acc[LIVE][TN] = {};
        const int m0 = wr * LIVE * 32, n0 = wc * TN * 32;               // first row and channel of the wavefront
        u32x4_t a[2][LIVE], b[2][TN];
        uint32_t asc[LIVE], bsc[TN], as_next[LIVE], bs_next[TN];
        const int swz = (r >> 2) & 3, at[2] = {(h ^ swz) * 16, ((2 + h) ^ swz) * 16};
        const uint8_t *a_lds = lds + (m0 + r) * 64, *b_lds = lds + BM * 64 + (n0 + r) * 64, *as_lds = lds + S::kCodes + (m0 + r) * 4, *bs_lds = lds + S::kCodes + (BM + n0 + r) * 4;
        auto read = [&](int stage, auto j_c) {                          // (stage: its place in LDS, in bytes)
            constexpr int J = decltype(j_c)::value;
#pragma unroll
            for (int n = 0; n < TN; ++n) b[J][n] = *reinterpret_cast<const u32x4_t *>(b_lds + at[J] + stage + n * 2048);
#pragma unroll
            for (int m = 0; m < LIVE; ++m) a[J][m] = *reinterpret_cast<const u32x4_t *>(a_lds + at[J] + stage + m * 2048);
        };
        auto read_scales = [&](int stage) {
#pragma unroll
            for (int n = 0; n < TN; ++n) bs_next[n] = *reinterpret_cast<const uint32_t *>(bs_lds + stage + n * 128);
#pragma unroll
            for (int m = 0; m < LIVE; ++m) as_next[m] = *reinterpret_cast<const uint32_t *>(as_lds + stage + m * 128);
        };
        auto take_scales = [&]() {                                      // bytes 0 and 2 are then this lane's in steps 0 and 1
#pragma unroll
            for (int n = 0; n < TN; ++n) bsc[n] = bs_next[n] >> (8 * h);
#pragma unroll
            for (int m = 0; m < LIVE; ++m) asc[m] = as_next[m] >> (8 * h);
        };
        auto multiply = [&](auto j_c) {
            constexpr int J = decltype(j_c)::value;
#pragma unroll
            for (int m = 0; m < LIVE; ++m)
#pragma unroll
                for (int n = 0; n < TN; ++n)
                    acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        i32x8_t{(int)b[J][n][0], (int)b[J][n][1], (int)b[J][n][2], (int)b[J][n][3], 0, 0, 0, 0},
                        i32x8_t{(int)a[J][m][0], (int)a[J][m][1], (int)a[J][m][2], (int)a[J][m][3], 0, 0, 0, 0}, acc[m][n], 4, 4, 2 * J, (int)bsc[n], 2 * J, (int)asc[m]);
        };
        constexpr std::integral_constant<int, 0> first{};
        constexpr std::integral_constant<int, 1> second{};
        // Every product's operands are read one step ahead of it: step 1's during step 0, the next stage's step 0 during step 1.  So stage s + 1 has to be
        // there in the middle of stage s; the stages after it may still be on their way.  The barrier there also says that everyone has read all of stage s,
        // whose place is refilled.  (hold(): left to itself the compiler moves step 0's products behind the barrier, where they wait with step 1's.)
        auto hold = [&]() {
#pragma unroll
            for (int m = 0; m < LIVE; ++m)
#pragma unroll
                for (int n = 0; n < TN; ++n) asm volatile("" : "+v"(acc[m][n]));
        };
        if (G >= NST) wait_loads<(NST - 2) * LA>();                     // (the first stages' weights came before all of their rows)
        else wait_loads<0>();
        __syncthreads();
        read(0, first);
        read_scales(0);
        int stage = 0;
        auto iterate = [&](int s, auto more_c) {
            const int next = stage + S::kStage == NST * S::kStage ? 0 : stage + S::kStage;
            read(stage, second);
            take_scales();
            multiply(first);
            hold();
            if constexpr (decltype(more_c)::value) wait_loads<(NST - 2) * L>();
            else wait_loads<0>();
            __syncthreads();
            read(next, first);
            read_scales(next);
            if constexpr (decltype(more_c)::value) issue_weights(s + NST, lds + stage), issue_rows(s + NST, lds + stage);
            multiply(second);
            hold();
            stage = next;
        };
        int s = 0;
        for (; s + NST < G; ++s) iterate(s, std::true_type{});
        for (; s + 1 < G; ++s) iterate(s, std::false_type{});
        if (4 * G - 2 < blocks) read(stage, second);
        take_scales();
        multiply(first);
        if (4 * G - 2 < blocks) multiply(second);
        __syncthreads();                                                // everyone is done with the ring
        uint8_t *patch = lds + wave * kMxPatch<OUT>;
        static_assert(TN % 2 == 0 && S::W * kMxPatch<OUT> <= S::kLds, "tiles leave in pairs, through the ring's place");
#pragma unroll
        for (int m = 0; m < LIVE; ++m) {
            const int i = m0 + 32 * m;
            if (i >= rows) break;
#pragma unroll
            for (int n = 0; n < TN; n += 2) {
                const int c = col * BN + n0 + 32 * n;
                if (c < N) mx_store_pair<OUT>(p, acc[m][n], acc[m][n + 1], e, c, row0 + i, rows - i, patch);
            }
        }
    };
    if (TM == 1 || live == 1) run(std::integral_constant<int, 1>{});
    else if (live == 2) run(std::integral_constant<int, TM < 2 ? TM : 2>{});
    else if (live == 3) run(std::integral_constant<int, TM < 3 ? TM : 3>{});
    else run(std::integral_constant<int, TM>{});
}

template <int WR, int WC, int TM, int TN, int NST>
static int launch_tile(const MxArgs &p, hipStream_t s)
{
    using S = MxTile<WR, WC, TM, TN, NST>;
    const long slots = (long)p.R / S::BM + (p.E < p.R ? p.E : p.R);
    const long wgs = (slots * ((p.N + S::BN - 1) / S::BN) + kXcds - 1) / kXcds * kXcds;      // upper bound of the work items, whole rounds of XCDs
    if (wgs * S::W > 0x3ffffff) return fail(MOE_ERR_UNSUPPORTED, "moe_grouped_gemm_mx4: %ld workgroups exceed one launch", wgs);
    auto run = [&](auto out) {
        constexpr int OUT = decltype(out)::value;
        static std::atomic<uint64_t> raised;
        raise_lds_limit(reinterpret_cast<const void *>(&mx4_tile_kernel<WR, WC, TM, TN, NST, OUT>), S::kLds, raised);
        hipLaunchKernelGGL((mx4_tile_kernel<WR, WC, TM, TN, NST, OUT>), dim3((unsigned)wgs), dim3(64 * S::W), S::kLds, s, p);
    };
    if (p.out_scales) run(std::integral_constant<int, -1>{});
    else if (p.out_dtype == MOE_F16) run(std::integral_constant<int, MOE_F16>{});
    else if (p.out_dtype == MOE_BF16) run(std::integral_constant<int, MOE_BF16>{});
    else run(std::integral_constant<int, MOE_F32>{});
    return check_launch("moe_grouped_gemm_mx4");
}

// Tiles of 128 rows by 256 channels, two blocks per compute unit, whose starts and ends overlap each other's loops (8192 tokens, two of 64 experts of 4096 x 16384: fc1 942 us,
// fc2 826; one block of 256 x 256 1065 and 786; 4096 tokens, two of 128 experts, 2048 x 8192, 281 and 359), and of 64 by 128 where that makes fewer than one
// and a half of them per compute unit (997 tokens, two of 16 experts of 704 x 2880: 15.3 + 11.5 us, 20.9 + 24.1 in large ones; 768, two of 32, 4096 x 1024: 19.5 and 26.6;
// left to large ones 1600, two of 32, 1024 x 4096: 25.5, small 32.4).
int launch_mx4_tiled(const MxArgs &p, hipStream_t s)
{
    return expected_row_tiles(p.most, p.E, 128) * ((p.N + 255) / 256) <= 384 ? launch_tile<2, 2, 1, 2, 3>(p, s) : launch_tile<1, 4, 4, 2, 3>(p, s);
}

}  // namespace moe
