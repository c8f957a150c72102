// Gated feed-forward block in bf16 on v_mfma_f32_32x32x16_bf16: tiles of G and U
// (BM rows of X against BF rows of Wg and the same BF rows of Wu).
//
// Staging.  All three operands are K-major per row, so a stage is BK columns
// of BM + 2 BF rows, copied straight to LDS (global_load_lds_dwordx4), NS
// stages deep.  A staged row holds BK / 8 pieces of 16 bytes; piece q of row r
// lies at piece q ^ f(r), so that the 16 rows that a quarter of a 16-byte LDS
// read covers fall into 16 different pieces of the 256-byte bank window.
// Operands are read one k-step (16 columns) ahead of the matrix instructions
// that take them.
//
// MFMA rows run over features and columns over positions, so a lane's four
// consecutive accumulators are four consecutive features of one position; G
// and U of a (position, feature) sit in the same lane and register, and H is
// formed there.  The results pass through LDS (each wave its own part) to be
// stored by whole 16-byte pieces of rows.
#include "ffn_bf16.hpp"

#include "ffn_tiles.hpp"

namespace dpg {
namespace {

// piece q of row r lies at piece q ^ swizzle(r)
__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

template <int BM_, int BF_, int WM_, int WF_, int BK_, int NS_>
struct Shape {
    static constexpr int BM = BM_, BF = BF_, WM = WM_, WF = WF_, BK = BK_, NS = NS_;
    static constexpr int WAVES = WM * WF, THREADS = 64 * WAVES;
    static constexpr int ROW = 2 * BK;                       // bytes of a staged row
    static constexpr int ROWS = BM + 2 * BF;
    static constexpr int STAGE = ROWS * ROW;
    static constexpr int RPI = 1024 / ROW;                   // rows per load instruction
    static constexpr int LOADS = ROWS / RPI / WAVES;         // per wave and stage
    static constexpr int FM = BM / WM / 32, FF = BF / WF / 32;
    static constexpr int LDS = NS * STAGE;
    static_assert(LOADS * RPI * WAVES == ROWS && BM % RPI == 0 && BF % RPI == 0, "stage split");
    static_assert(WAVES * 32 * (FF * 128 + 16) <= LDS, "the output transpose fits the stages");
    static_assert(NS >= 2 && NS <= 4, "waits");
    static_assert(BK == 64, "eight pieces in a row; two sets of operands in turn");
};

template <typename S, int ACT>
__global__ __launch_bounds__(S::THREADS, 1) void ffn_forward_kernel(const uint16_t *__restrict__ X,
                                                                    const uint16_t *__restrict__ Wg,
                                                                    const uint16_t *__restrict__ Wu, i64 M, i64 K, i64 F,
                                                                    int tiles_m, int tiles_f, uint16_t *__restrict__ H,
                                                                    uint16_t *__restrict__ G,
                                                                    uint16_t *__restrict__ U, int vec)
{
    typedef uint16_t T;
    constexpr int FM = S::FM, FF = S::FF, BK = S::BK, NS = S::NS, ROW = S::ROW, KS = BK / 16;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    int tm, tf;
    tile_of((int)blockIdx.x, (int)gridDim.x, tiles_m, tiles_f, tm, tf);
    const i64 m0 = (i64)tm * S::BM, f0 = (i64)tf * S::BF;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WF * (FM * 32), wf = wave % S::WF * (FF * 32);
    const uint32_t lds0 = lds_addr(smem);
    const int nst = (int)((K + BK - 1) / BK);
    const int tail = (int)(K - (i64)(nst - 1) * BK);         // columns of the last stage

    // the wave's loads of a stage: rows past the end read the last row (their products are not stored)
    const char *base[S::LOADS];
    uint32_t off[S::LOADS];
    int q[S::LOADS];
#pragma unroll
    for (int r = 0; r < S::LOADS; ++r) {
        const int row = (wave + S::WAVES * r) * S::RPI + lane / (64 / S::RPI);
        const int first = __builtin_amdgcn_readfirstlane(row);
        const uint16_t *P = first < S::BM ? X + m0 * K : first < S::BM + S::BF ? Wg + f0 * K : Wu + f0 * K;
        const int in = first < S::BM ? row : first < S::BM + S::BF ? row - S::BM : row - S::BM - S::BF;
        const i64 left = first < S::BM ? M - m0 : F - f0;
        base[r] = reinterpret_cast<const char *>(P);
        q[r] = (lane % (64 / S::RPI)) ^ swizzle(row);
        off[r] = (uint32_t)(in < left ? in : (int)left - 1) * (uint32_t)(2 * K) + 16u * q[r];
    }
    const auto issue = [&](int c) {
        const uint32_t L = lds0 + (uint32_t)(c % NS) * S::STAGE;
        const bool cut = c == nst - 1 && tail < BK;
#pragma unroll
        for (int r = 0; r < S::LOADS; ++r)
            // columns past the end read the stage's first ones, and are zeroed in LDS
            dma16_off(base[r] + (i64)c * (2 * BK), cut && 8 * q[r] >= tail ? off[r] - 16u * q[r] : off[r],
                      L + 1024 * (wave + S::WAVES * r));
    };
    const auto zero_tail = [&](int c) {
        if (c != nst - 1 || tail == BK) return;
        char *L = smem + (c % NS) * S::STAGE;
#pragma unroll
        for (int r = 0; r < S::LOADS; ++r)
            if (8 * q[r] >= tail)
                *reinterpret_cast<uint4 *>(L + 1024 * (wave + S::WAVES * r) + 16 * lane) = make_uint4(0, 0, 0, 0);
    };

    f32x16_t ag[FM][FF], au[FM][FF];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FF; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) ag[x][y][r] = au[x][y][r] = 0.0f;

    struct Frag {
        bf16x8_t x[FM], g[FF], u[FF];
    };
    const int li = lane & 31, lk = lane >> 5;
    const int sw = swizzle(li);                          // of every row li + 32 n
    const auto load_frag = [&](const char *L, int ks, Frag &f) {
        const int at = 16 * ((2 * ks + lk) ^ sw) + li * ROW;
#pragma unroll
        for (int x = 0; x < FM; ++x)
            f.x[x] = *reinterpret_cast<const bf16x8_t *>(L + (wm + 32 * x) * ROW + at);
#pragma unroll
        for (int y = 0; y < FF; ++y) {
            f.g[y] = *reinterpret_cast<const bf16x8_t *>(L + (S::BM + wf + 32 * y) * ROW + at);
            f.u[y] = *reinterpret_cast<const bf16x8_t *>(L + (S::BM + S::BF + wf + 32 * y) * ROW + at);
        }
    };
    const auto mma = [&](const Frag &f) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FF; ++y) {
                ag[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.g[y], f.x[x], ag[x][y], 0, 0, 0);
                au[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.u[y], f.x[x], au[x][y], 0, 0, 0);
            }
    };
    // a k-step's operand reads between its matrix instructions
    const auto interleave = [&]() {
        constexpr int reads = FM + 2 * FF, mfma = 2 * FM * FF, per = (reads + mfma - 1) / mfma;
#pragma unroll
        for (int i = 0; i < reads / per; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);       // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, per, 0);     // LDS reads
        }
        __builtin_amdgcn_sched_group_barrier(0x100, reads % per, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, mfma - reads / per, 0);
    };

#pragma unroll
    for (int c = 0; c < NS - 1; ++c)
        if (c < nst) issue(c);
    {
        const int later = (nst < NS - 1 ? nst : NS - 1) - 1;
        wait_stages_after<S::LOADS>(later);
        zero_tail(0);
        wait_lgkmcnt0();
        stage_barrier();
        if (NS - 1 < nst) issue(NS - 1);
    }
    // every trip is one straight run of blocks, so that the accumulators stay where they are: the last stage is peeled
    Frag fa, fb;
    load_frag(smem, 0, fa);
    const auto inside = [&](const char *L) {
#pragma unroll
        for (int ks = 0; ks + 1 < KS; ++ks) {
            load_frag(L, ks + 1, (ks & 1) == 0 ? fb : fa);
            mma((ks & 1) == 0 ? fa : fb);
            interleave();
        }
    };
    for (int c = 0; c + 1 < nst; ++c) {
        inside(smem + (c % NS) * S::STAGE);
        // stage c + 1 has landed, and every wave has read the last of stage c: its buffer takes stage c + NS
        wait_stages_after<S::LOADS>(nst - 2 - c < NS - 2 ? nst - 2 - c : NS - 2);
        zero_tail(c + 1);
        wait_lgkmcnt0();
        stage_barrier();
        if (c + NS < nst) issue(c + NS);
        load_frag(smem + ((c + 1) % NS) * S::STAGE, 0, fa);
        mma(fb);
        interleave();
    }
    inside(smem + ((nst - 1) % NS) * S::STAGE);
    mma(fb);
    __syncthreads();                                         // the stages become the output transposes

    constexpr int LDT = FF * 32 * (int)sizeof(T) + 16;
    char *L = smem + wave * 32 * LDT;
    const auto put = [&](int x, auto value, T *O) {
#pragma unroll
        for (int y = 0; y < FF; ++y)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
                put4(reinterpret_cast<T *>(L + li * LDT) + 32 * y + 8 * rb + 4 * lk, value(y, 4 * rb),
                     value(y, 4 * rb + 1), value(y, 4 * rb + 2), value(y, 4 * rb + 3));
        store_rows<T, FF * 32, LDT>(L, O, M, F, m0 + wm + 32 * x, f0 + wf, vec != 0, lane);
    };
#pragma unroll
    for (int x = 0; x < FM; ++x) {
        put(x, [&](int y, int r) { return act_for<ACT, T>(ag[x][y][r]) * au[x][y][r]; }, H);
        if (G != nullptr) {
            put(x, [&](int y, int r) { return ag[x][y][r]; }, G);
            put(x, [&](int y, int r) { return au[x][y][r]; }, U);
        }
    }
}

template <typename S>
void launch_forward(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, dp_act act,
                    uint16_t *H, uint16_t *G, uint16_t *U, hipStream_t stream)
{
    const int tm = (int)ceil_div(M, S::BM), tf = (int)ceil_div(F, S::BF);
    const int vec = F % 8 == 0 && aligned(H, 16) && aligned(G, 16) && aligned(U, 16);
    const unsigned grid = (unsigned)((i64)tm * tf);
    if (act == DP_ACT_SILU)
        ffn_forward_kernel<S, DP_ACT_SILU><<<grid, S::THREADS, 0, stream>>>(X, Wg, Wu, M, K, F, tm, tf, H, G, U, vec);
    else
        ffn_forward_kernel<S, DP_ACT_GELU_TANH><<<grid, S::THREADS, 0, stream>>>(X, Wg, Wu, M, K, F, tm, tf, H, G, U,
                                                                                 vec);
}

// ---------------------------------------------------------------------------
// dX = BG Wg + BU Wu: one product whose K runs over BG's features, then BU's.
// BG and BU are staged as X above; Wg and Wu lie K-major ([feature][d_in]),
// so their operands come from transposing LDS reads (bf16_stage.hpp).
// With several splits each takes a run of the stages and writes fp32 partial
// tiles, which a second kernel adds in split order.
// ---------------------------------------------------------------------------
template <int BM_, int BD_, int WM_, int WD_, int BK_, int NS_>
struct DxShape {
    static constexpr int BM = BM_, BD = BD_, WM = WM_, WD = WD_, BK = BK_, NS = NS_;
    static constexpr int WAVES = WM * WD, THREADS = 64 * WAVES;
    static constexpr int A_ROW = 2 * BK, W_ROW = 2 * BD;         // bytes of a staged row
    static constexpr int A_BYTES = BM * A_ROW, W_BYTES = BK * W_ROW, STAGE = A_BYTES + W_BYTES;
    static constexpr int A_RPI = 1024 / A_ROW, W_RPI = 1024 / W_ROW;
    static constexpr int A_LOADS = A_BYTES / 1024 / WAVES, W_LOADS = W_BYTES / 1024 / WAVES, LOADS = A_LOADS + W_LOADS;
    static constexpr int FM = BM / WM / 32, FD = BD / WD / 32;
    static constexpr int LDS = NS * STAGE;
    static_assert(A_LOADS * WAVES * 1024 == A_BYTES && W_LOADS * WAVES * 1024 == W_BYTES, "stage split");
    static_assert(BK == 64, "eight pieces in a row; two sets of operands in turn");
    static_assert(WAVES * 32 * (FD * 128 + 16) <= LDS, "the output transpose fits the stages");
};

template <typename S, bool SPLIT>
__global__ __launch_bounds__(S::THREADS, 1) void ffn_dx_kernel(const uint16_t *__restrict__ BG,
                                                               const uint16_t *__restrict__ BU,
                                                               const uint16_t *__restrict__ Wg,
                                                               const uint16_t *__restrict__ Wu, i64 M, i64 D, i64 F,
                                                               i64 lda, i64 ldw, int tiles_m, int tiles_d, int splits,
                                                               uint16_t *__restrict__ dX, float *__restrict__ part,
                                                               int vec)
{
    typedef uint16_t T;
    constexpr int FM = S::FM, FD = S::FD, BK = S::BK, NS = S::NS, KS = BK / 16;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    int tm, td;
    const int tiles = tiles_m * tiles_d, split = SPLIT ? (int)blockIdx.x / tiles : 0;
    tile_of((int)blockIdx.x - split * tiles, tiles, tiles_m, tiles_d, tm, td);
    const i64 m0 = (i64)tm * S::BM, d0 = (i64)td * S::BD;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WD * (FM * 32), wd = wave % S::WD * (FD * 32);
    const uint32_t lds0 = lds_addr(smem);
    const int half = (int)((F + BK - 1) / BK);               // stages of each product
    const int tail = (int)(F - (i64)(half - 1) * BK);        // rows of W (columns of B) in the last of them
    const int first = SPLIT ? (int)((i64)split * 2 * half / splits) : 0;
    const int nst = (SPLIT ? (int)((i64)(split + 1) * 2 * half / splits) : 2 * half) - first;

    uint32_t offA[S::A_LOADS], offW[S::W_LOADS];
    int q[S::A_LOADS], kr[S::W_LOADS];
#pragma unroll
    for (int r = 0; r < S::A_LOADS; ++r) {
        const int row = (wave + S::WAVES * r) * S::A_RPI + lane / (64 / S::A_RPI);
        q[r] = (lane % (64 / S::A_RPI)) ^ swizzle(row);
        offA[r] = (uint32_t)(row < M - m0 ? row : (int)(M - m0) - 1) * (uint32_t)(2 * lda) + 16u * q[r];
    }
#pragma unroll
    for (int r = 0; r < S::W_LOADS; ++r) {
        kr[r] = (wave + S::WAVES * r) * S::W_RPI + lane / (64 / S::W_RPI);
        const i64 d = 8 * ((lane % (64 / S::W_RPI)) ^ (4 * (kr[r] & 3)));
        offW[r] = (uint32_t)kr[r] * (uint32_t)(2 * ldw) + (uint32_t)(2 * (d0 + d < ldw ? d : ldw - 8 - d0));
    }
    const auto issue = [&](int c) {
        const uint32_t L = lds0 + (uint32_t)(c % NS) * S::STAGE;
        const int g = first + c, run = g >= half, k = g - run * half;
        const bool cut = k == half - 1 && tail < BK;
        const char *a = reinterpret_cast<const char *>((run ? BU : BG) + m0 * lda) + (i64)k * (2 * BK);
        const char *w = reinterpret_cast<const char *>((run ? Wu : Wg) + (i64)k * BK * ldw + d0);
#pragma unroll
        for (int r = 0; r < S::A_LOADS; ++r)
            dma16_off(a, cut && 8 * q[r] >= tail ? offA[r] - 16u * q[r] : offA[r], L + 1024 * (wave + S::WAVES * r));
#pragma unroll
        for (int r = 0; r < S::W_LOADS; ++r)
            // (one row of tiles reads each weight once)
            dma16_off<(S::BM <= 64)>(w, cut && kr[r] >= tail ? offW[r] - (uint32_t)kr[r] * (uint32_t)(2 * ldw) : offW[r],
                      L + S::A_BYTES + 1024 * (wave + S::WAVES * r));
    };
    // features past the end read the stage's first ones, and are zeroed in LDS on both sides
    const auto zero_tail = [&](int c) {
        const int g = first + c, k = g >= half ? g - half : g;
        if (k != half - 1 || tail == BK) return;
        char *L = smem + (c % NS) * S::STAGE;
#pragma unroll
        for (int r = 0; r < S::A_LOADS; ++r)
            if (8 * q[r] >= tail)
                *reinterpret_cast<uint4 *>(L + 1024 * (wave + S::WAVES * r) + 16 * lane) = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < S::W_LOADS; ++r)
            if (kr[r] >= tail)
                *reinterpret_cast<uint4 *>(L + S::A_BYTES + 1024 * (wave + S::WAVES * r) + 16 * lane) =
                    make_uint4(0, 0, 0, 0);
    };

    f32x16_t acc[FM][FD];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FD; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.0f;

    struct Frag {
        bf16x8_t a[FM], w[FD];
    };
    const int li = lane & 31, lk = lane >> 5;
    const int sw = swizzle(li);
    const auto load_frag = [&](const char *L, int ks, Frag &f) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
            f.a[x] = *reinterpret_cast<const bf16x8_t *>(L + (wm + 32 * x + li) * S::A_ROW + 16 * ((2 * ks + lk) ^ sw));
#pragma unroll
        for (int y = 0; y < FD; ++y) f.w[y] = read_operand(L + S::A_BYTES, S::W_ROW, 16 * ks, wd + 32 * y, lane);
    };
    const auto mma = [&](const Frag &f) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FD; ++y)
                acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.w[y], f.a[x], acc[x][y], 0, 0, 0);
    };
    const auto interleave = [&]() {
        constexpr int reads = FM + 2 * FD, mfma = FM * FD, per = (reads + mfma - 1) / mfma;
#pragma unroll
        for (int i = 0; i < reads / per; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, per, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, reads % per, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, mfma - reads / per, 0);
    };

#pragma unroll
    for (int c = 0; c < NS - 1; ++c)
        if (c < nst) issue(c);
    wait_stages_after<S::LOADS>((nst < NS - 1 ? nst : NS - 1) - 1);
    zero_tail(0);
    wait_lgkmcnt0();
    stage_barrier();
    if (NS - 1 < nst) issue(NS - 1);
    Frag fa, fb;
    load_frag(smem, 0, fa);
    const auto inside = [&](const char *L) {
#pragma unroll
        for (int ks = 0; ks + 1 < KS; ++ks) {
            load_frag(L, ks + 1, (ks & 1) == 0 ? fb : fa);
            mma((ks & 1) == 0 ? fa : fb);
            interleave();
        }
    };
    for (int c = 0; c + 1 < nst; ++c) {
        inside(smem + (c % NS) * S::STAGE);
        wait_stages_after<S::LOADS>(nst - 2 - c < NS - 2 ? nst - 2 - c : NS - 2);
        zero_tail(c + 1);
        wait_lgkmcnt0();
        stage_barrier();
        if (c + NS < nst) issue(c + NS);
        load_frag(smem + ((c + 1) % NS) * S::STAGE, 0, fa);
        mma(fb);
        interleave();
    }
    inside(smem + ((nst - 1) % NS) * S::STAGE);
    mma(fb);

    if constexpr (SPLIT) {
        float *P = part + (i64)split * M * ldw;
#pragma unroll
        for (int x = 0; x < FM; ++x)
#pragma unroll
            for (int y = 0; y < FD; ++y)
#pragma unroll
                for (int rb = 0; rb < 4; ++rb) {
                    const i64 m = m0 + wm + 32 * x + li, d = d0 + wd + 32 * y + 8 * rb + 4 * lk;
                    if (m < M && d < ldw)                    // ldw % 8 == 0: the four are all in or all out
                        *reinterpret_cast<float4 *>(P + m * ldw + d) =
                            make_float4(acc[x][y][4 * rb], acc[x][y][4 * rb + 1], acc[x][y][4 * rb + 2],
                                        acc[x][y][4 * rb + 3]);
                }
        return;
    }
    __syncthreads();
    constexpr int LDT = FD * 32 * (int)sizeof(T) + 16;
    char *L = smem + wave * 32 * LDT;
#pragma unroll
    for (int x = 0; x < FM; ++x) {
#pragma unroll
        for (int y = 0; y < FD; ++y)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
                put4(reinterpret_cast<T *>(L + li * LDT) + 32 * y + 8 * rb + 4 * lk, acc[x][y][4 * rb],
                     acc[x][y][4 * rb + 1], acc[x][y][4 * rb + 2], acc[x][y][4 * rb + 3]);
        store_rows<T, FD * 32, LDT>(L, dX, M, D, m0 + wm + 32 * x, d0 + wd, vec != 0, lane);
    }
}

// dX = the splits' partial sums, in split order; rows of ld (a multiple of 4) there, of D here
__global__ __launch_bounds__(256) void ffn_dx_sum_kernel(const float *__restrict__ part, i64 M, i64 D, i64 ld,
                                                         int splits, uint16_t *__restrict__ dX)
{
    const i64 n = M * ld;
    for (i64 i = ((i64)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (i64)gridDim.x * 1024) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < splits; k += 8) {
            float4 p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                p[j] = k + j < splits ? *reinterpret_cast<const float4 *>(part + (i64)(k + j) * n + i)
                                      : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[0] += p[j].x;
                v[1] += p[j].y;
                v[2] += p[j].z;
                v[3] += p[j].w;
            }
        }
        const i64 m = D == ld ? 0 : i / ld, d = i - m * ld;  // D = ld: one row of all values
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (D == ld || d + j < D) store_elem(dX + m * D + d + j, v[j]);
    }
}

typedef DxShape<256, 256, 2, 4, 64, 2> LargeDx;
typedef DxShape<128, 128, 2, 2, 64, 4> MidDx;
typedef DxShape<64, 128, 1, 4, 64, 3> Rows64Dx;
typedef DxShape<32, 128, 1, 4, 64, 3> Rows32Dx;

template <typename S>
void launch_dx(const uint16_t *BG, const uint16_t *BU, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 D, i64 F,
               i64 lda, i64 ldw, int splits, uint16_t *dX, float *part, hipStream_t stream)
{
    const int tm = (int)ceil_div(M, S::BM), td = (int)ceil_div(D, S::BD);
    const int vec = D % 8 == 0 && aligned(dX, 16);
    const unsigned grid = (unsigned)((i64)tm * td * splits);
    if (splits == 1) {
        ffn_dx_kernel<S, false><<<grid, S::THREADS, 0, stream>>>(BG, BU, Wg, Wu, M, D, F, lda, ldw, tm, td, 1, dX, nullptr,
                                                                 vec);
        return;
    }
    ffn_dx_kernel<S, true><<<grid, S::THREADS, 0, stream>>>(BG, BU, Wg, Wu, M, D, F, lda, ldw, tm, td, splits, dX, part,
                                                            vec);
    const i64 blocks = ceil_div(M * ldw, 1024);
    ffn_dx_sum_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, stream>>>(part, M, D, ldw, splits, dX);
}

size_t pad_bytes(i64 rows, i64 cols)
{
    return cols % 8 == 0 ? 0 : align_up(sizeof(uint16_t) * (size_t)(rows * padded(cols)), 256);
}

// Arrays whose rows are padded to 16 bytes: [rows][cols] into rows of
// padded(cols), zeros behind.  One launch for all of a call's (pieces of eight
// values, first[k] the first of array k).
struct Pads {
    int count;
    const uint16_t *P[4];
    uint16_t *O[4];
    i64 cols[4], first[5];
};

__global__ __launch_bounds__(256) void ffn_pad_kernel(Pads s)
{
    for (i64 i = (i64)blockIdx.x * 256 + threadIdx.x; i < s.first[s.count]; i += (i64)gridDim.x * 256) {
        int k = 0;
        while (k + 1 < s.count && i >= s.first[k + 1]) ++k;
        const i64 cols = s.cols[k], per = (cols + 7) / 8, j = i - s.first[k], r = j / per, c = (j - r * per) * 8;
        const uint16_t *p = s.P[k] + r * cols + c;
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t a = c + 2 * q < cols ? p[2 * q] : 0, b = c + 2 * q + 1 < cols ? p[2 * q + 1] : 0;
            w[q] = a | (b << 16);
        }
        *reinterpret_cast<uint4 *>(s.O[k] + 8 * j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Adds P to the arrays to pad, if its rows need it; returns where its rows are
// then (in the workspace at ws, which is moved on, or in P itself).
const uint16_t *pad_rows(Pads &s, const uint16_t *P, i64 rows, i64 cols, char *&ws)
{
    if (cols % 8 == 0) return P;
    const int k = s.count++;
    s.P[k] = P;
    s.O[k] = (uint16_t *)ws;
    s.cols[k] = cols;
    s.first[k + 1] = s.first[k] + rows * (padded(cols) / 8);
    ws += pad_bytes(rows, cols);
    return s.O[k];
}

void pad(const Pads &s, hipStream_t stream)
{
    if (s.count == 0) return;
    const i64 blocks = ceil_div(s.first[s.count], 256);
    ffn_pad_kernel<<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, stream>>>(s);
}

enum { kRows32, kRows64, kMid, kLarge };

struct DxPlan {
    int shape, splits;
};

// Tile shape and splits by the time they take: rounds of 256 workgroups, each
// of its stages at what one takes (256 x 256 tiles 1.75 us, 128 x 128 0.59:
// measured at 8192 x 11008 -> 4096 and 4096 x 2048 -> 768 alone, and taken for
// all sizes), and the partial tiles written and read.  4096 x 2048 -> 768 (192 tiles of 128): 53 us in one
// split, 65 in two; 128 x 11008 -> 4096 (32 tiles): 206 us in one, 64 in eight.
DxPlan dx_plan(i64 M, i64 D, i64 F)
{
    const i64 stages = 2 * ceil_div(F, 64);
    DxPlan p = {kMid, 1};
    if (M <= 64) {                        // one row of tiles: the weights' bytes bound it, over two workgroups per CU
        p.shape = M <= 32 ? kRows32 : kRows64;
        i64 most = 512 / ceil_div(D, 128);
        if (most > stages / 4) most = stages / 4;
        if (most > 32) most = 32;
        // one stage after another at 0.5 us, or one more launch, and the partial tiles beside the weights (16 x 512 ->
        // 256: 10.7 us in one split, 13.1 in four; 16 x 1024 -> 1024: 17.4 and 13.1; 64 x 4096 -> 4096: 67 in one, 24.5
        // in eight, 28 in sixteen)
        double best = 0.5 * (double)stages;
        for (int s = 2; s <= most; ++s) {
            const double t = 0.5 * (double)ceil_div(stages, s) + 7.0 + 16.0 * s * (double)M * (double)D / 4.5e6;
            if (t < best) {
                best = t;
                p.splits = s;
            }
        }
        return p;
    }
    double best = 1e30;
    for (int shape = kMid; shape <= kLarge; ++shape) {
        const i64 b = shape == kLarge ? 256 : 128, tiles = ceil_div(M, b) * ceil_div(D, b);
        for (int s = 1; s <= 16 && s <= stages / 4 + 1; ++s) {
            const double t = (double)ceil_div(tiles * s, 256) * (double)ceil_div(stages, s) * (shape == kLarge ? 1.75 : 0.59) +
                             (s > 1 ? 4.0 + 8.0 * s * (double)M * (double)D / 4.5e6 : 0.0);
            if (t < best) {
                best = t;
                p.shape = shape;
                p.splits = s;
            }
        }
    }
    return p;
}

typedef Shape<256, 128, 4, 2, 64, 2> Large;
typedef Shape<128, 64, 2, 2, 64, 2> Mid;       // two workgroups per CU
typedef Shape<128, 64, 2, 2, 64, 4> Deep;      // one
typedef Shape<64, 64, 2, 2, 64, 4> Rows64;

// Tiles by the rounds that they take: 256 large ones, or 512 middle ones, at
// 0.64 of the time (4096 x 1024 -> 2752, 352 large tiles: 60.3 us large, 59.3
// middle; 4096 x 768 -> 2048, 256 tiles: 30.5 and 37.3); up to 256 middle ones
// run one to a CU with four stages in flight (128 x 4096 -> 11008: 53.3 us,
// 64.5 with two).
enum { kTilesRows64, kTilesDeep, kTilesMid, kTilesLarge };
int forward_tiles(i64 M, i64 F)
{
    if (M <= 64) return kTilesRows64;
    const i64 large = ceil_div(M, 256) * ceil_div(F, 128), mid = ceil_div(M, 128) * ceil_div(F, 64);
    if ((double)ceil_div(large, 256) <= 0.64 * (double)ceil_div(mid, 512)) return kTilesLarge;
    return mid <= 256 ? kTilesDeep : kTilesMid;
}

}  // namespace

size_t ffn_bf16_forward_workspace(i64 M, i64 K, i64 F) { return pad_bytes(M, K) + 2 * pad_bytes(F, K); }

void ffn_bf16_forward(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, dp_act act,
                      uint16_t *H, uint16_t *G, uint16_t *U, void *ws, hipStream_t stream)
{
    char *w = (char *)ws;
    Pads s = {};
    X = pad_rows(s, X, M, K, w);
    Wg = pad_rows(s, Wg, F, K, w);
    Wu = pad_rows(s, Wu, F, K, w);
    pad(s, stream);
    K = padded(K);
    const int tiles = forward_tiles(M, F);
    if (tiles == kTilesLarge) launch_forward<Large>(X, Wg, Wu, M, K, F, act, H, G, U, stream);
    else if (tiles == kTilesMid) launch_forward<Mid>(X, Wg, Wu, M, K, F, act, H, G, U, stream);
    else if (tiles == kTilesDeep) launch_forward<Deep>(X, Wg, Wu, M, K, F, act, H, G, U, stream);
    else launch_forward<Rows64>(X, Wg, Wu, M, K, F, act, H, G, U, stream);
}

size_t ffn_bf16_dx_workspace(i64 M, i64 D, i64 F)
{
    const DxPlan p = dx_plan(M, D, F);
    const size_t part = p.splits > 1 ? sizeof(float) * (size_t)p.splits * (size_t)(M * padded(D)) : 0;
    return 2 * pad_bytes(M, F) + 2 * pad_bytes(F, D) + part;
}

void ffn_bf16_dx(const uint16_t *BG, const uint16_t *BU, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 D, i64 F,
                 uint16_t *dX, void *ws, hipStream_t stream)
{
    const DxPlan p = dx_plan(M, D, F);
    char *w = (char *)ws;
    Pads s = {};
    BG = pad_rows(s, BG, M, F, w);
    BU = pad_rows(s, BU, M, F, w);
    Wg = pad_rows(s, Wg, F, D, w);
    Wu = pad_rows(s, Wu, F, D, w);
    pad(s, stream);
    const i64 lda = padded(F), ldw = padded(D);
    float *part = (float *)w;
    if (p.shape == kLarge) launch_dx<LargeDx>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, stream);
    else if (p.shape == kMid) launch_dx<MidDx>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, stream);
    else if (p.shape == kRows64) launch_dx<Rows64Dx>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, stream);
    else launch_dx<Rows32Dx>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, stream);
}

}  // namespace dpg
