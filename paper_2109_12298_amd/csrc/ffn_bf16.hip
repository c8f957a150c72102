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

#include "bf16_stage.hpp"
#include "ffn_any.hpp"

namespace dpg {
namespace {

using namespace bf16s;
using namespace ffn;

// lane l's 16 bytes at base + off go to LDS byte lds + 16 l (see dma16); STREAM:
// past the caches
template <bool STREAM = false>
__device__ __forceinline__ void dma16_off(const void *base, uint32_t off, uint32_t lds)
{
    if constexpr (STREAM)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base),
                     "s"(__builtin_amdgcn_readfirstlane(lds))
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base),
                     "s"(__builtin_amdgcn_readfirstlane(lds))
                     : "memory", "m0");
}

// wait until all but the last `later` (at most 2) stages' loads have landed, N loads each
template <int N>
__device__ __forceinline__ void wait_later(int later)
{
    if (later >= 2) wait_vmcnt<2 * N>();
    else if (later == 1) wait_vmcnt<N>();
    else wait_vmcnt<0>();
}

template <int BK>
__device__ __forceinline__ int swizzle(int row)
{
    return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
}

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
    static_assert(BK / 16 % 2 == 0, "two sets of operands in turn");
};

// Tile order: workgroups go round robin over the XCDs; each XCD takes a run of
// consecutive tiles, 8 tiles of positions by as many tiles of features as the
// run holds, so that its L2 serves the operand rows that they share.
__device__ __forceinline__ void tile_of(int b, int nb, int tiles_m, int tiles_n, int &tm, int &tn)
{
    constexpr int GM = 8;
    const int t = (int)xcd_swizzle32((uint32_t)b, (uint32_t)nb);
    const int group = t / (GM * tiles_n), m0 = group * GM;
    const int gm = tiles_m - m0 < GM ? tiles_m - m0 : GM;
    const int in = t - group * GM * tiles_n;
    tm = m0 + in % gm;
    tn = in / gm;
}

// 32 rows by COLS values of one output tile, from LDS rows of LDT bytes
template <typename T, int COLS, int LDT>
__device__ __forceinline__ void store_rows(const char *L, T *__restrict__ O, i64 rows, i64 cols, i64 r0, i64 c0, bool vec,
                                           int lane)
{
    if (vec) {                            // 16-byte pieces
        constexpr int N = 16 / sizeof(T), LPR = COLS / N, RPS = 64 / LPR;    // values per piece, lanes per row, rows per store
#pragma unroll
        for (int s = 0; s < 32 / RPS; ++s) {
            const int row = s * RPS + lane / LPR, c = lane % LPR;
            const uint4 v = *reinterpret_cast<const uint4 *>(L + row * LDT + 16 * c);
            const i64 r = r0 + row, f = c0 + N * c;
            if (r < rows && f < cols) *reinterpret_cast<uint4 *>(O + r * cols + f) = v;
        }
    } else {                              // rows of any alignment: 64 consecutive values per store
#pragma unroll 8
        for (int s = 0; s < 32 * COLS / 64; ++s) {
            const int row = (64 * s + lane) / COLS, c = (64 * s + lane) % COLS;
            const T v = *reinterpret_cast<const T *>(L + row * LDT + (int)sizeof(T) * c);
            const i64 r = r0 + row, f = c0 + c;
            if (r < rows && f < cols) O[r * cols + f] = v;
        }
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    return (uint32_t)bf16_bits(a) | ((uint32_t)bf16_bits(b) << 16);
}

// four consecutive values of a row to LDS
__device__ __forceinline__ void put4(uint16_t *p, float a, float b, float c, float d)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(a, b), pack2(c, d));
}
__device__ __forceinline__ void put4(float *p, float a, float b, float c, float d)
{
    *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d);
}

// The products of an fp32 contraction from three bf16 parts of each operand
// (x = x0 + x1 + x2, exact; see ffn_split_kernel), smallest first: part s of
// the list is x's part X_PART >> 2 s & 3 times w's part W_PART >> 2 s & 3.
// Left out are x1 w2, x2 w1 (2^-24 of the product at most) and x2 w2.
constexpr uint32_t X_PART = 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10;
constexpr uint32_t W_PART = 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10;
constexpr int kParts = 6;

// What the kernels of an fp32 call need besides the parts: the values
// themselves (K features in a row), and a word per workgroup of the splitting
// kernel that is not 0 where it met a value without parts.
struct Whole {
    const float *a, *b, *wg, *wu;         // X (b unused), or BG and BU
    i64 K;
    const int32_t *flags;
    int count;
};

// whether any of the words is set, in every thread of the workgroup
__device__ __forceinline__ bool any_flag(const Whole &w)
{
    int bad = 0;
    for (int i = threadIdx.x; i < w.count; i += blockDim.x) bad |= w.flags[i];
    return __syncthreads_or(bad) != 0;
}

// T = float: X, Wg and Wu are the three parts of each ([3][rows][K], K a
// multiple of BK).
template <typename S, int ACT, typename T>
__global__ __launch_bounds__(S::THREADS, 1) void ffn_forward_kernel(const uint16_t *__restrict__ X,
                                                                    const uint16_t *__restrict__ Wg,
                                                                    const uint16_t *__restrict__ Wu, i64 M, i64 K, i64 F,
                                                                    int tiles_m, int tiles_f, T *__restrict__ H,
                                                                    T *__restrict__ G, T *__restrict__ U, int vec,
                                                                    Whole whole)
{
    constexpr bool PARTS = sizeof(T) == 4;
    constexpr int FM = S::FM, FF = S::FF, BK = S::BK, NS = S::NS, ROW = S::ROW, KS = BK / 16;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    int tm, tf;
    tile_of((int)blockIdx.x, (int)gridDim.x, tiles_m, tiles_f, tm, tf);
    const i64 m0 = (i64)tm * S::BM, f0 = (i64)tf * S::BF;
    if constexpr (PARTS) {
        if (any_flag(whole)) {
            for (int t = 0; t < (S::BM / kTM) * (S::BF / kTN); ++t)
                any_forward_tile<S::THREADS, ACT>(whole.a, whole.wg, whole.wu, M, whole.K, F,
                                                  m0 + t / (S::BF / kTN) * kTM, f0 + t % (S::BF / kTN) * kTN, H, G, U,
                                                  reinterpret_cast<float *>(smem));
            return;
        }
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WF * (FM * 32), wf = wave % S::WF * (FF * 32);
    const uint32_t lds0 = lds_addr(smem);
    const int per = (int)((K + BK - 1) / BK);
    const int nst = PARTS ? kParts * per : per;
    const int tail = (int)(K - (i64)(per - 1) * BK);         // columns of the last stage

    // the wave's loads of a stage: rows past the end read the last row (their products are not stored)
    const char *base[S::LOADS];
    uint32_t off[S::LOADS];
    int q[S::LOADS];
    bool is_x[S::LOADS];
#pragma unroll
    for (int r = 0; r < S::LOADS; ++r) {
        const int row = (wave + S::WAVES * r) * S::RPI + lane / (64 / S::RPI);
        const int first = __builtin_amdgcn_readfirstlane(row);
        const uint16_t *P = first < S::BM ? X + m0 * K : first < S::BM + S::BF ? Wg + f0 * K : Wu + f0 * K;
        const int in = first < S::BM ? row : first < S::BM + S::BF ? row - S::BM : row - S::BM - S::BF;
        const i64 left = first < S::BM ? M - m0 : F - f0;
        base[r] = reinterpret_cast<const char *>(P);
        is_x[r] = first < S::BM;
        q[r] = (lane % (64 / S::RPI)) ^ swizzle<BK>(row);
        off[r] = (uint32_t)(in < left ? in : (int)left - 1) * (uint32_t)(2 * K) + 16u * q[r];
    }
    const auto issue = [&](int c) {
        const uint32_t L = lds0 + (uint32_t)(c % NS) * S::STAGE;
        const bool cut = !PARTS && c == nst - 1 && tail < BK;
        i64 xo = (i64)c * (2 * BK), wo = xo;
        if (PARTS) {
            const int p = c / per;
            const i64 k = (i64)(c - p * per) * (2 * BK);
            xo = k + (i64)((X_PART >> (2 * p)) & 3) * (2 * M * K);
            wo = k + (i64)((W_PART >> (2 * p)) & 3) * (2 * F * K);
        }
#pragma unroll
        for (int r = 0; r < S::LOADS; ++r)
            // columns past the end read the stage's first ones, and are zeroed in LDS
            dma16_off(base[r] + (is_x[r] ? xo : wo), cut && 8 * q[r] >= tail ? off[r] - 16u * q[r] : off[r],
                      L + 1024 * (wave + S::WAVES * r));
    };
    const auto zero_tail = [&](int c) {
        if (PARTS || c != nst - 1 || tail == BK) return;
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
    const int sw = swizzle<BK>(li);                          // of every row li + 32 n
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
        wait_later<S::LOADS>(later);
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
        wait_later<S::LOADS>(nst - 2 - c < NS - 2 ? nst - 2 - c : NS - 2);
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

template <typename S, typename T>
void launch_forward(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, dp_act act, T *H,
                    T *G, T *U, const Whole &whole, hipStream_t stream)
{
    const int tm = (int)ceil_div(M, S::BM), tf = (int)ceil_div(F, S::BF);
    const int vec = F * sizeof(T) % 16 == 0 && aligned(H, 16) && aligned(G, 16) && aligned(U, 16);
    const unsigned grid = (unsigned)((i64)tm * tf);
    if (act == DP_ACT_SILU)
        ffn_forward_kernel<S, DP_ACT_SILU, T><<<grid, S::THREADS, 0, stream>>>(X, Wg, Wu, M, K, F, tm, tf, H, G, U, vec,
                                                                               whole);
    else
        ffn_forward_kernel<S, DP_ACT_GELU_TANH, T><<<grid, S::THREADS, 0, stream>>>(X, Wg, Wu, M, K, F, tm, tf, H, G, U,
                                                                                    vec, whole);
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
    static_assert(WAVES * 32 * (FD * 128 + 16) <= LDS, "the output transpose fits the stages");
};

// T = float: BG and Wg point to the parts of both products ([2][3][M][lda] and
// [2][3][F][ldw], F = lda a multiple of BK), BU and Wu are not used.
template <typename S, bool SPLIT, typename T>
__global__ __launch_bounds__(S::THREADS, 1) void ffn_dx_kernel(const uint16_t *__restrict__ BG,
                                                               const uint16_t *__restrict__ BU,
                                                               const uint16_t *__restrict__ Wg,
                                                               const uint16_t *__restrict__ Wu, i64 M, i64 D, i64 F,
                                                               i64 lda, i64 ldw, int tiles_m, int tiles_d, int splits,
                                                               T *__restrict__ dX, float *__restrict__ part, int vec,
                                                               Whole whole)
{
    constexpr bool PARTS = sizeof(T) == 4;
    constexpr int RUNS = PARTS ? 2 * kParts : 2;             // products that the stages run through
    constexpr int FM = S::FM, FD = S::FD, BK = S::BK, NS = S::NS, KS = BK / 16;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    int tm, td;
    const int tiles = tiles_m * tiles_d, split = SPLIT ? (int)blockIdx.x / tiles : 0;
    tile_of((int)blockIdx.x - split * tiles, tiles, tiles_m, tiles_d, tm, td);
    const i64 m0 = (i64)tm * S::BM, d0 = (i64)td * S::BD;
    if constexpr (PARTS) {
        if (any_flag(whole)) {
            if (split == 0)
                for (int t = 0; t < (S::BM / kTM) * (S::BD / kTN); ++t)
                    any_dx_tile<S::THREADS>(whole.a, whole.b, whole.wg, whole.wu, M, D, whole.K,
                                            m0 + t / (S::BD / kTN) * kTM, d0 + t % (S::BD / kTN) * kTN, dX,
                                            reinterpret_cast<float *>(smem));
            return;
        }
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WD * (FM * 32), wd = wave % S::WD * (FD * 32);
    const uint32_t lds0 = lds_addr(smem);
    const int half = (int)((F + BK - 1) / BK);               // stages of each product
    const int tail = (int)(F - (i64)(half - 1) * BK);        // rows of W (columns of B) in the last of them
    const int first = SPLIT ? (int)((i64)split * RUNS * half / splits) : 0;
    const int nst = (SPLIT ? (int)((i64)(split + 1) * RUNS * half / splits) : RUNS * half) - first;

    uint32_t offA[S::A_LOADS], offW[S::W_LOADS];
    int q[S::A_LOADS], kr[S::W_LOADS];
#pragma unroll
    for (int r = 0; r < S::A_LOADS; ++r) {
        const int row = (wave + S::WAVES * r) * S::A_RPI + lane / (64 / S::A_RPI);
        q[r] = (lane % (64 / S::A_RPI)) ^ swizzle<BK>(row);
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
        const int g = first + c, run = PARTS ? g / half : g >= half, k = g - run * half;
        const bool cut = !PARTS && k == half - 1 && tail < BK;
        const uint16_t *ab = run ? BU : BG, *wb = run ? Wu : Wg;
        if (PARTS) {
            const int u = run >= kParts, p = 2 * (u ? run - kParts : run);
            ab = BG + (3 * u + (int)((X_PART >> p) & 3)) * (M * lda);
            wb = Wg + (3 * u + (int)((W_PART >> p) & 3)) * (F * ldw);
        }
        const char *a = reinterpret_cast<const char *>(ab + m0 * lda) + (i64)k * (2 * BK);
        const char *w = reinterpret_cast<const char *>(wb + (i64)k * BK * ldw + d0);
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
        if (PARTS || k != half - 1 || tail == BK) return;
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
    const int sw = swizzle<BK>(li);
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
    wait_later<S::LOADS>((nst < NS - 1 ? nst : NS - 1) - 1);
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
        wait_later<S::LOADS>(nst - 2 - c < NS - 2 ? nst - 2 - c : NS - 2);
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
template <typename T>
__global__ __launch_bounds__(256) void ffn_dx_sum_kernel(const float *__restrict__ part, i64 M, i64 D, i64 ld,
                                                         int splits, T *__restrict__ dX, Whole whole)
{
    if (sizeof(T) == 4 && any_flag(whole)) return;           // dX is there already
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

template <typename S, typename T>
void launch_dx(const uint16_t *BG, const uint16_t *BU, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 D, i64 F,
               i64 lda, i64 ldw, int splits, T *dX, float *part, const Whole &whole, hipStream_t stream)
{
    const int tm = (int)ceil_div(M, S::BM), td = (int)ceil_div(D, S::BD);
    const int vec = D * sizeof(T) % 16 == 0 && aligned(dX, 16);
    const unsigned grid = (unsigned)((i64)tm * td * splits);
    if (splits == 1) {
        ffn_dx_kernel<S, false, T><<<grid, S::THREADS, 0, stream>>>(BG, BU, Wg, Wu, M, D, F, lda, ldw, tm, td, 1, dX,
                                                                    nullptr, vec, whole);
        return;
    }
    ffn_dx_kernel<S, true, T><<<grid, S::THREADS, 0, stream>>>(BG, BU, Wg, Wu, M, D, F, lda, ldw, tm, td, splits, dX,
                                                               part, vec, whole);
    const i64 blocks = ceil_div(M * ldw, 1024);
    ffn_dx_sum_kernel<T><<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, stream>>>(part, M, D, ldw, splits, dX,
                                                                                        whole);
}

i64 padded(i64 cols) { return (cols + 7) / 8 * 8; }

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
// measured at 8192 x 11008 -> 4096 and 4096 x 2048 -> 768), and the partial
// tiles written and read.  4096 x 2048 -> 768 (192 tiles of 128): 53 us in one
// split, 65 in two; 128 x 11008 -> 4096 (32 tiles): 206 us in one, 64 in eight.
// runs: products of F features that the stages run through (2, or 12 for fp32 in parts)
DxPlan dx_plan(i64 M, i64 D, i64 F, int runs)
{
    const i64 stages = runs * ceil_div(F, 64);
    DxPlan p = {kMid, 1};
    if (M <= 64) {                        // one row of tiles: the weights' bytes bound it, over two workgroups per CU
        p.shape = M <= 32 ? kRows32 : kRows64;
        i64 s = 512 / ceil_div(D, 128);
        if (s > stages / 4) s = stages / 4;
        if (s > 32) s = 32;
        p.splits = s < 1 ? 1 : (int)s;
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

template <typename T>
void forward_by_tiles(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, dp_act act, T *H,
                      T *G, T *U, const Whole &whole, hipStream_t stream)
{
    const int tiles = forward_tiles(M, F);
    if (tiles == kTilesLarge) launch_forward<Large, T>(X, Wg, Wu, M, K, F, act, H, G, U, whole, stream);
    else if (tiles == kTilesMid) launch_forward<Mid, T>(X, Wg, Wu, M, K, F, act, H, G, U, whole, stream);
    else if (tiles == kTilesDeep) launch_forward<Deep, T>(X, Wg, Wu, M, K, F, act, H, G, U, whole, stream);
    else if constexpr (sizeof(T) == 2) launch_forward<Rows64, T>(X, Wg, Wu, M, K, F, act, H, G, U, whole, stream);
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
    forward_by_tiles<uint16_t>(X, Wg, Wu, M, K, F, act, H, G, U, Whole{}, stream);
}

size_t ffn_bf16_dx_workspace(i64 M, i64 D, i64 F)
{
    const DxPlan p = dx_plan(M, D, F, 2);
    const size_t part = p.splits > 1 ? sizeof(float) * (size_t)p.splits * (size_t)(M * padded(D)) : 0;
    return 2 * pad_bytes(M, F) + 2 * pad_bytes(F, D) + part;
}

void ffn_bf16_dx(const uint16_t *BG, const uint16_t *BU, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 D, i64 F,
                 uint16_t *dX, void *ws, hipStream_t stream)
{
    const DxPlan p = dx_plan(M, D, F, 2);
    char *w = (char *)ws;
    Pads s = {};
    BG = pad_rows(s, BG, M, F, w);
    BU = pad_rows(s, BU, M, F, w);
    Wg = pad_rows(s, Wg, F, D, w);
    Wu = pad_rows(s, Wu, F, D, w);
    pad(s, stream);
    const i64 lda = padded(F), ldw = padded(D);
    float *part = (float *)w;
    if (p.shape == kLarge) launch_dx<LargeDx, uint16_t>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, Whole{}, stream);
    else if (p.shape == kMid) launch_dx<MidDx, uint16_t>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, Whole{}, stream);
    else if (p.shape == kRows64) launch_dx<Rows64Dx, uint16_t>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, Whole{}, stream);
    else launch_dx<Rows32Dx, uint16_t>(BG, BU, Wg, Wu, M, D, F, lda, ldw, p.splits, dX, part, Whole{}, stream);
}

// ---------------------------------------------------------------------------
// fp32 by parts
// ---------------------------------------------------------------------------
namespace {

constexpr i64 kAlignK = 64;               // a whole stage
i64 whole(i64 n) { return (n + kAlignK - 1) / kAlignK * kAlignK; }

// x = p[0] + p[1] + p[2] exactly, each a bf16 value (8 bits each, rounded to
// nearest, so that what the left-out products hold has no preferred sign).
// Returns true where that fails: infinities and NaN, values so large that
// they round to infinity, and values under 2^-100, whose last bits may lie
// below the smallest normal bf16, which the matrix unit takes as zero.
__device__ __forceinline__ bool split3(float x, uint32_t (&p)[3])
{
    const uint32_t e = (__float_as_uint(x) >> 23) & 255u;
    p[0] = bf16_bits(x);
    const float r1 = x - bf16_to_f32((uint16_t)p[0]);
    p[1] = bf16_bits(r1);
    p[2] = bf16_bits(r1 - bf16_to_f32((uint16_t)p[1]));
    return x != 0.0f && (e >= 254u || e < 27u);
}

// Arrays to split: P [rows][cols] as O [3][rows_out][ld], zeros past rows and
// cols.  One launch for all of a call's (pieces of eight values, first[k] the
// first of array k), of at most kSplitBlocks workgroups, each leaving a word
// that says whether it met a value that cannot be split.
constexpr int kSplitBlocks = 1024;

struct Splits {
    int count;
    const float *P[4];
    uint16_t *O[4];
    i64 rows[4], cols[4], ld[4], plane[4], first[5];
};

__global__ __launch_bounds__(256) void ffn_split_kernel(Splits s, int32_t *__restrict__ flags)
{
    bool bad = false;
    for (i64 i = (i64)blockIdx.x * 256 + threadIdx.x; i < s.first[s.count]; i += (i64)gridDim.x * 256) {
        int k = 0;
        while (k + 1 < s.count && i >= s.first[k + 1]) ++k;
        const i64 rows = s.rows[k], cols = s.cols[k], per = s.ld[k] / 8;
        const i64 j = i - s.first[k], r = j / per, c = (j - r * per) * 8;
        const float *p = s.P[k] + r * cols + c;
        float x[8];
        if (cols % 4 == 0 && (reinterpret_cast<uintptr_t>(s.P[k]) & 15) == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = r < rows && c + 4 * h < cols;
                const float4 v = in ? *reinterpret_cast<const float4 *>(p + 4 * h) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = r < rows && c + q < cols ? p[q] : 0.0f;
        }
        uint32_t w[3][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t a[3], b[3];
            bad |= split3(x[2 * q], a);
            bad |= split3(x[2 * q + 1], b);
#pragma unroll
            for (int n = 0; n < 3; ++n) w[n][q] = a[n] | (b[n] << 16);
        }
#pragma unroll
        for (int n = 0; n < 3; ++n)
            *reinterpret_cast<uint4 *>(s.O[k] + n * s.plane[k] + 8 * j) = make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]);
    }
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) flags[blockIdx.x] = any;
}

constexpr size_t kFlagBytes = sizeof(int32_t) * kSplitBlocks;

void add_split(Splits &s, const float *P, i64 rows, i64 cols, i64 rows_out, i64 ld, uint16_t *O)
{
    const int k = s.count++;
    s.P[k] = P;
    s.O[k] = O;
    s.rows[k] = rows;
    s.cols[k] = cols;
    s.ld[k] = ld;
    s.plane[k] = rows_out * ld;
    s.first[k + 1] = s.first[k] + rows_out * (ld / 8);
}

// Splits the arrays; returns how many words were left at flags.
int split(const Splits &s, int32_t *flags, hipStream_t stream)
{
    const i64 blocks = ceil_div(s.first[s.count], 256);
    const int n = (int)(blocks < kSplitBlocks ? blocks : kSplitBlocks);
    ffn_split_kernel<<<(unsigned)n, 256, 0, stream>>>(s, flags);
    return n;
}

size_t part_bytes(i64 rows, i64 ld) { return align_up(3 * sizeof(uint16_t) * (size_t)(rows * ld), 256); }

}  // namespace

size_t ffn_parts_forward_workspace(i64 M, i64 K, i64 F)
{
    return kFlagBytes + part_bytes(M, whole(K)) + 2 * part_bytes(F, whole(K));
}

void ffn_parts_forward(const float *X, const float *Wg, const float *Wu, i64 M, i64 K, i64 F, dp_act act, float *H,
                       float *G, float *U, void *ws, hipStream_t stream)
{
    const i64 ld = whole(K);
    int32_t *flags = (int32_t *)ws;
    uint16_t *x = (uint16_t *)((char *)ws + kFlagBytes);
    uint16_t *g = (uint16_t *)((char *)x + part_bytes(M, ld)), *u = (uint16_t *)((char *)g + part_bytes(F, ld));
    Splits s = {};
    add_split(s, X, M, K, M, ld, x);
    add_split(s, Wg, F, K, F, ld, g);
    add_split(s, Wu, F, K, F, ld, u);
    const int n = split(s, flags, stream);
    forward_by_tiles<float>(x, g, u, M, ld, F, act, H, G, U, Whole{X, nullptr, Wg, Wu, K, flags, n}, stream);
}

size_t ffn_parts_dx_workspace(i64 M, i64 D, i64 F)
{
    const DxPlan p = dx_plan(M, D, whole(F), 2 * kParts);
    const i64 lda = whole(F), ldw = padded(D);
    const size_t part = p.splits > 1 ? sizeof(float) * (size_t)p.splits * (size_t)(M * ldw) : 0;
    return kFlagBytes + align_up(6 * sizeof(uint16_t) * (size_t)(M * lda), 256) +
           align_up(6 * sizeof(uint16_t) * (size_t)(lda * ldw), 256) + part;
}

void ffn_parts_dx(const float *BG, const float *BU, const float *Wg, const float *Wu, i64 M, i64 D, i64 F, float *dX,
                  void *ws, hipStream_t stream)
{
    const i64 lda = whole(F), ldw = padded(D);
    const DxPlan p = dx_plan(M, D, lda, 2 * kParts);
    int32_t *flags = (int32_t *)ws;
    uint16_t *b = (uint16_t *)((char *)ws + kFlagBytes);
    uint16_t *w = (uint16_t *)((char *)b + align_up(6 * sizeof(uint16_t) * (size_t)(M * lda), 256));
    float *part = (float *)((char *)w + align_up(6 * sizeof(uint16_t) * (size_t)(lda * ldw), 256));
    Splits s = {};
    add_split(s, BG, M, F, M, lda, b);
    add_split(s, BU, M, F, M, lda, b + 3 * M * lda);
    add_split(s, Wg, F, D, lda, ldw, w);
    add_split(s, Wu, F, D, lda, ldw, w + 3 * lda * ldw);
    const Whole whole_ = {BG, BU, Wg, Wu, F, flags, split(s, flags, stream)};
    if (p.shape == kLarge)
        launch_dx<LargeDx, float>(b, nullptr, w, nullptr, M, D, lda, lda, ldw, p.splits, dX, part, whole_, stream);
    else launch_dx<MidDx, float>(b, nullptr, w, nullptr, M, D, lda, lda, ldw, p.splits, dX, part, whole_, stream);
}

}  // namespace dpg
