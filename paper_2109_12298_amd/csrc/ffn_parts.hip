// Gated feed-forward block in fp32 on v_mfma_f32_32x32x16_bf16: every value as
// three bf16 parts (split_bf16.hpp), every product as six bf16 products
//   x w = x0 w2 + x2 w0 + x1 w1 + x0 w1 + x1 w0 + x0 w0
// added in fp32 in this order.  What is left out (x1 w2, x2 w1: 2^-24 of the
// product at most, and x2 w2) is within the rounding of an fp32 product.  The
// parts are those of 2^24 x, so that a value of any size has normal ones and
// small values beside ordinary ones cost nothing (GELU's slopes end at 2^-100
// and below); 2^-48 comes out of the sums.
//
// Infinities, NaN, values whose parts overflow (from about 2^104 on) and sums
// that do (from 2^80 on) leave non-finite sums.  A workgroup that finds one
// among its own forms its tile again on the fp32 units (ffn_any.hpp): the other
// tiles keep their bits and their time.  Such a tile is slow, single loads and
// no overlap: with one NaN in dH, 512 x 2752 -> 1024 takes 684 us instead of 61.
//
// A stage holds 16 columns of all three parts of each operand, so that a part
// is staged once and read from LDS once for all the products that take it: 12
// operand reads for 24 matrix instructions.  (Products one after another, each
// with stages of its own, take 32 reads for 24, and twice the loads: 4096 x
// 2048 -> 5504 with the split 974 us, 850 so; 1000 x 500 -> 1333 44 and 32.)
// Two workgroups of four waves share a CU and cover each other's first loads
// and last stores; stages of 32 columns, one workgroup per CU, take 911 and 34.
// The first of these sizes runs at about 1.4 PFLOP/s, a large library product's
// rate; small ones are bound by the split (6 us) and the stages' latency.
//
// Operands and the output's way are those of ffn_bf16.hip.
#include "ffn_any.hpp"
#include "ffn_bf16.hpp"
#include "ffn_tiles.hpp"
#include "split_bf16.hpp"

#include <type_traits>

namespace dpg {
namespace {

constexpr int kBK = 16, kNS = 3, kPlanes = 3, kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRow = 2 * kBK;             // bytes of a staged row of X, Wg, Wu, BG or BU
constexpr int kRpi = 1024 / kRow;         // such rows per load instruction
constexpr int kCols = 128;                // columns of a staged row of Wg and Wu in the backward pass
constexpr int kWRpi = 1024 / (2 * kCols); // such rows per load instruction
constexpr int kWLoads = kBK / kWRpi;      // load instructions per part and stage
constexpr int kSplitBlocks = 1024;        // workgroups of the splitting kernel, at most
constexpr int kSumRows = 16;              // rows by kTN columns of a workgroup that adds splits
constexpr int kProducts = 6;
constexpr int kXPart[kProducts] = {0, 2, 1, 0, 1, 0}, kWPart[kProducts] = {2, 0, 1, 1, 0, 0};

// The operands themselves, for tiles that are formed again: X (b unused), or BG
// and BU, with K features in a row.
struct Whole {
    const float *a, *b, *wg, *wu;
    i64 K;
};

// 0, or NaN where a value is not finite
__device__ __forceinline__ float probe(const f32x16_t &v)
{
    float t = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(v[r], 0.0f, t);
    return t;
}

// The parts lie in memory as they do in LDS: a load instruction copies 1 KB of
// consecutive bytes (pieces of rows, parts of cache lines, of a row-major array:
// 4096 x 2048 -> 5504 1343 us).  Rows of X, Wg, Wu, BG and BU: [group of kRpi
// rows][stage][part] of 1 KB.
struct Parts {
    const char *p;
    i64 groups, stages;
    __device__ __forceinline__ const char *at(i64 group, i64 part) const
    {
        return p + ((group < groups ? group : groups - 1) * stages * kPlanes + part) * 1024;
    }
};
constexpr i64 kStageBytes = kPlanes * 1024;                  // from a group's stage to its next

constexpr int kOperands = 12;             // of a wave and k-step
constexpr int kMfma = 24;                 // matrix instructions of a wave and k-step
constexpr int kLoads = 6;                 // loads of a wave and stage

// Where a staged row holds columns 8 q .. 8 q + 7: the 16 rows that a quarter of a 16-byte LDS read covers fall into 16
// different pieces of the 256-byte bank window.
__device__ __forceinline__ int piece_of(int row, int q) { return q ^ ((row >> 3) & 1); }

// The run of stages 0 .. nst-1, a stage being one k-step.  issue(c, r): load r
// of stage c; read(c, j, f): operand j of stage c; mma(i, f): matrix
// instruction i.  The loads and reads of what comes next are issued in the
// shadow of the matrix instructions (32 clocks each), in this order.
template <typename Frag, typename Issue, typename Read, typename Mma>
__device__ __forceinline__ void run_stages(int nst, const Issue &issue, const Read &read, const Mma &mma)
{
    static_assert(kNS == 3, "two stages ahead");
#pragma unroll
    for (int c = 0; c < kNS; ++c)
        if (c < nst)
#pragma unroll
            for (int r = 0; r < kLoads; ++r) issue(c, r);
    wait_stages_after<kLoads>(nst - 1);
    stage_barrier();
    Frag fa, fb;
#pragma unroll
    for (int j = 0; j < kOperands; ++j) read(0, j, fa);
    // f: stage c's operands, next: those of stage c + 1
    const auto step = [&](auto ISSUE, int c, const Frag &f, Frag &next) {
        // stage c + 1 has landed, and every wave has read stage c: its buffer takes stage c + kNS
        if constexpr (decltype(ISSUE)::value) wait_vmcnt<kLoads>();
        else wait_stages_after<kLoads>(nst - 2 - c < 1 ? 0 : 1);
        wait_lgkmcnt0();
        stage_barrier();
        if constexpr (!decltype(ISSUE)::value)
            if (c + kNS < nst)
#pragma unroll
                for (int r = 0; r < kLoads; ++r) issue(c + kNS, r);
#pragma unroll
        for (int i = 0; i < kMfma; ++i) {
            mma(i, f);
            if (i < kOperands) read(c + 1, i, next);
            if constexpr (decltype(ISSUE)::value)
                if (i % (kMfma / kLoads) == 1) issue(c + kNS, i / (kMfma / kLoads));
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto last = [&](const Frag &f) {
#pragma unroll
        for (int i = 0; i < kMfma; ++i) mma(i, f);
    };
    int c = 0;
    for (; c + 1 + kNS < nst; c += 2) {
        step(std::true_type(), c, fa, fb);
        step(std::true_type(), c + 1, fb, fa);
    }
    for (;; c += 2) {
        if (c + 1 == nst) {
            last(fa);
            return;
        }
        step(std::false_type(), c, fa, fb);
        if (c + 2 == nst) {
            last(fb);
            return;
        }
        step(std::false_type(), c + 1, fb, fa);
    }
}

// ---------------------------------------------------------------------------
// forward: tiles of BM positions by BF features of both G and U, each wave half
// of either
// ---------------------------------------------------------------------------
template <int BM_, int BF_>
struct Shape {
    static constexpr int BM = BM_, BF = BF_, ROWS = BM + 2 * BF;
    static constexpr int STAGE = kPlanes * ROWS * kRow, LDS = kNS * STAGE;
    static constexpr int LOADS = kPlanes * ROWS / kRpi / kWaves;
    static constexpr int FM = BM / 64, FF = BF / 64;
    static_assert(kPlanes * (FM + 2 * FF) == kOperands && kProducts * 2 * FM * FF == kMfma && LOADS == kLoads, "steps");
    static_assert(LOADS * kRpi * kWaves == kPlanes * ROWS && BM % kRpi == 0 && BF % kRpi == 0, "stage split");
    static_assert(kWaves * 32 * (FF * 128 + 16) <= LDS && 4 * kAnyFloats <= LDS, "the outputs' and the fallback's LDS");
};

template <typename S, int ACT>
__global__ __launch_bounds__(kThreads, 2) void ffn_parts_forward_kernel(Parts X, Parts Wg, Parts Wu, i64 M, i64 F,
                                                                        int tiles_m, int tiles_f,
                                                                        float *__restrict__ H, float *__restrict__ G,
                                                                        float *__restrict__ U, int vec, Whole whole)
{
    constexpr int FM = S::FM, FF = S::FF;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    int tm, tf;
    tile_of((int)blockIdx.x, (int)gridDim.x, tiles_m, tiles_f, tm, tf);
    const i64 m0 = (i64)tm * S::BM, f0 = (i64)tf * S::BF;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / 2 * (FM * 32), wf = wave % 2 * (FF * 32);
    const uint32_t lds0 = lds_addr(smem);

    // the wave's loads of a stage: [part][group of rows] of X, then of Wg, then of Wu; groups past the end read the last
    // one (their products are not stored)
    const char *base[S::LOADS];
#pragma unroll
    for (int r = 0; r < S::LOADS; ++r) {
        const int i = wave + kWaves * r;
        constexpr int GX = S::BM / kRpi, GW = S::BF / kRpi;
        if (i < kPlanes * GX) {
            base[r] = X.at(m0 / kRpi + i % GX, i / GX);
        } else {
            const int w = i - kPlanes * GX, v = w < kPlanes * GW ? w : w - kPlanes * GW;
            base[r] = (w < kPlanes * GW ? Wg : Wu).at(f0 / kRpi + v % GW, v / GW);
        }
    }
    f32x16_t ag[FM][FF], au[FM][FF];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FF; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) ag[x][y][r] = au[x][y][r] = 0.0f;

    struct Frag {
        bf16x8_t x[kPlanes][FM], g[kPlanes][FF], u[kPlanes][FF];
    };
    const int li = lane & 31, lk = lane >> 5;
    const int at = li * kRow + 16 * piece_of(li, lk);
    const auto issue = [&](int c, int r) {
        dma16_off(base[r] + c * kStageBytes, 16u * lane, lds0 + (uint32_t)(c % kNS) * S::STAGE + 1024 * (wave + kWaves * r));
    };
    const auto read = [&](int c, int j, Frag &f) {
        const char *L = smem + (c % kNS) * S::STAGE + at;
        const int p = j % kPlanes, n = j / kPlanes;
        if (n < FM) {
            f.x[p][n] = *reinterpret_cast<const bf16x8_t *>(L + (p * S::BM + wm + 32 * n) * kRow);
        } else if (n < FM + FF) {
            f.g[p][n - FM] =
                *reinterpret_cast<const bf16x8_t *>(L + (kPlanes * S::BM + p * S::BF + wf + 32 * (n - FM)) * kRow);
        } else {
            f.u[p][n - FM - FF] = *reinterpret_cast<const bf16x8_t *>(
                L + (kPlanes * (S::BM + S::BF) + p * S::BF + wf + 32 * (n - FM - FF)) * kRow);
        }
    };
    const auto mma = [&](int i, const Frag &f) {
        const int n = i / (2 * FM * FF), x = i / 2 / FF % FM, y = i / 2 % FF;
        if (i % 2 == 0) {
            f32x16_t &g = ag[x][y];
            g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.g[kWPart[n]][y], f.x[kXPart[n]][x], g, 0, 0, 0);
        } else {
            f32x16_t &u = au[x][y];
            u = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.u[kWPart[n]][y], f.x[kXPart[n]][x], u, 0, 0, 0);
        }
    };
    run_stages<Frag>((int)X.stages, issue, read, mma);
    float sums = 0.0f;
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FF; ++y) sums += probe(ag[x][y]) + probe(au[x][y]);
    if (__syncthreads_or(sums != 0.0f)) {                    // the stages are free from here on
        for (int t = 0; t < (S::BM / kTM) * (S::BF / kTN); ++t)
            any_forward_tile<kThreads, ACT>(whole.a, whole.wg, whole.wu, M, whole.K, F, m0 + t / (S::BF / kTN) * kTM,
                                            f0 + t % (S::BF / kTN) * kTN, H, G, U, reinterpret_cast<float *>(smem));
        return;
    }
    // the stages become the output transposes
    constexpr int LDT = FF * 128 + 16;
    char *L = smem + wave * 32 * LDT;
    const auto put = [&](int x, auto value, float *O) {
#pragma unroll
        for (int y = 0; y < FF; ++y)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
                put4(reinterpret_cast<float *>(L + li * LDT) + 32 * y + 8 * rb + 4 * lk, value(y, 4 * rb),
                     value(y, 4 * rb + 1), value(y, 4 * rb + 2), value(y, 4 * rb + 3));
        store_rows<float, FF * 32, LDT>(L, O, M, F, m0 + wm + 32 * x, f0 + wf, vec != 0, lane);
    };
#pragma unroll
    for (int x = 0; x < FM; ++x) {
        const auto g = [&](int y, int r) { return ag[x][y][r] * split::kUnscale; };
        const auto u = [&](int y, int r) { return au[x][y][r] * split::kUnscale; };
        put(x, [&](int y, int r) { return act_for<ACT, float>(g(y, r)) * u(y, r); }, H);
        if (G != nullptr) {
            put(x, g, G);
            put(x, u, U);
        }
    }
}

typedef Shape<128, 64> Tile;

// ---------------------------------------------------------------------------
// dX = BG Wg + BU Wu: tiles of 128 positions by 128 columns, the stages through
// both products' features, with several splits each a run of them.
// W: the parts of Wg, then of Wu, each [block of kCols columns][stage][part][rows
// of the stage], kCols columns of a row.
// ---------------------------------------------------------------------------
struct DxTile {
    static constexpr int BM = 128, BD = kCols, W_ROW = 2 * BD;
    static constexpr int A_BYTES = kPlanes * BM * kRow, W_PLANE = kBK * W_ROW, W_BYTES = kPlanes * W_PLANE;
    static constexpr int STAGE = A_BYTES + W_BYTES, LDS = kNS * STAGE;
    static constexpr int A_LOADS = A_BYTES / 1024 / kWaves, W_LOADS = W_BYTES / 1024 / kWaves, LOADS = A_LOADS + W_LOADS;
    static constexpr int FM = BM / 64, FD = BD / 64;
    static_assert(kPlanes * (FM + FD) == kOperands && kProducts * FM * FD == kMfma && LOADS == kLoads, "steps");
    static_assert(A_LOADS * kWaves * 1024 == A_BYTES && W_LOADS * kWaves * 1024 == W_BYTES, "stage split");
    static_assert(kWaves * 32 * (FD * 128 + 16) <= LDS && 4 * kAnyFloats <= LDS, "the outputs' and the fallback's LDS");
};

template <bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void ffn_parts_dx_kernel(Parts BG, Parts BU, const char *__restrict__ W, i64 M,
                                                                   i64 D, i64 ldw, int tiles_m, int tiles_d, int splits,
                                                                   float *__restrict__ dX, float *__restrict__ part,
                                                                   int vec, Whole whole)
{
    typedef DxTile S;
    constexpr int FM = S::FM, FD = S::FD;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    int tm, td;
    const int tiles = tiles_m * tiles_d, split = SPLIT ? (int)blockIdx.x / tiles : 0;
    tile_of((int)blockIdx.x - split * tiles, tiles, tiles_m, tiles_d, tm, td);
    const i64 m0 = (i64)tm * S::BM, d0 = (i64)td * S::BD;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / 2 * (FM * 32), wd = wave % 2 * (FD * 32);
    const uint32_t lds0 = lds_addr(smem);
    const int half = (int)BG.stages;                         // of each product
    const int first = SPLIT ? (int)((i64)split * 2 * half / splits) : 0;
    const int nst = (SPLIT ? (int)((i64)(split + 1) * 2 * half / splits) : 2 * half) - first;

    // groups past the end read the last one (their products are not stored, and what is not finite among them is so in
    // the tile's own rows)
    const char *baseA[2][S::A_LOADS];
#pragma unroll
    for (int r = 0; r < S::A_LOADS; ++r) {
        constexpr int GA = S::BM / kRpi;
        const int i = wave + kWaves * r;
        baseA[0][r] = BG.at(m0 / kRpi + i % GA, i / GA);
        baseA[1][r] = BU.at(m0 / kRpi + i % GA, i / GA);
    }
    const i64 w_run = (i64)tiles_d * half * S::W_BYTES;
    const char *baseW = W + (i64)td * half * S::W_BYTES + 1024 * wave;
    f32x16_t acc[FM][FD];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FD; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.0f;

    struct Frag {
        bf16x8_t a[kPlanes][FM], w[kPlanes][FD];
    };
    const int li = lane & 31, lk = lane >> 5;
    const int at = li * kRow + 16 * piece_of(li, lk);
    const auto issue = [&](int c, int r) {
        const uint32_t L = lds0 + (uint32_t)(c % kNS) * S::STAGE;
        const int g = first + c, run = g >= half, k = g - run * half;
        if (r < S::A_LOADS)
            dma16_off((run ? baseA[1][r] : baseA[0][r]) + k * kStageBytes, 16u * lane, L + 1024 * (wave + kWaves * r));
        else
            dma16_off(baseW + run * w_run + (i64)k * S::W_BYTES + 1024 * kWaves * (r - S::A_LOADS), 16u * lane,
                      L + S::A_BYTES + 1024 * (wave + kWaves * (r - S::A_LOADS)));
    };
    const auto read = [&](int c, int j, Frag &f) {
        const char *L = smem + (c % kNS) * S::STAGE;
        const int p = j % kPlanes, n = j / kPlanes;
        if (n < FM)
            f.a[p][n] = *reinterpret_cast<const bf16x8_t *>(L + (p * S::BM + wm + 32 * n) * kRow + at);
        else
            f.w[p][n - FM] = read_operand(L + S::A_BYTES + p * S::W_PLANE, S::W_ROW, 0, wd + 32 * (n - FM), lane);
    };
    const auto mma = [&](int i, const Frag &f) {
        const int n = i / (FM * FD), x = i / FD % FM, y = i % FD;
        f32x16_t &a = acc[x][y];
        a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.w[kWPart[n]][y], f.a[kXPart[n]][x], a, 0, 0, 0);
    };
    run_stages<Frag>(nst, issue, read, mma);
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
                        put4(P + m * ldw + d, acc[x][y][4 * rb], acc[x][y][4 * rb + 1], acc[x][y][4 * rb + 2],
                             acc[x][y][4 * rb + 3]);
                }
        return;
    }
    float sums = 0.0f;
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FD; ++y) sums += probe(acc[x][y]);
    if (__syncthreads_or(sums != 0.0f)) {                    // the stages are free from here on
        for (int t = 0; t < (S::BM / kTM) * (S::BD / kTN); ++t)
            any_dx_tile<kThreads>(whole.a, whole.b, whole.wg, whole.wu, M, D, whole.K, m0 + t / (S::BD / kTN) * kTM,
                                  d0 + t % (S::BD / kTN) * kTN, dX, reinterpret_cast<float *>(smem));
        return;
    }
    constexpr int LDT = FD * 128 + 16;
    char *L = smem + wave * 32 * LDT;
#pragma unroll
    for (int x = 0; x < FM; ++x) {
#pragma unroll
        for (int y = 0; y < FD; ++y)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
                put4(reinterpret_cast<float *>(L + li * LDT) + 32 * y + 8 * rb + 4 * lk,
                     acc[x][y][4 * rb] * split::kUnscale, acc[x][y][4 * rb + 1] * split::kUnscale,
                     acc[x][y][4 * rb + 2] * split::kUnscale, acc[x][y][4 * rb + 3] * split::kUnscale);
        store_rows<float, FD * 32, LDT>(L, dX, M, D, m0 + wm + 32 * x, d0 + wd, vec != 0, lane);
    }
}

// dX = the splits' partial sums (times 2^48; rows of ld, a multiple of 8) in split order; a workgroup takes kSumRows rows
// by kTN columns, and forms them again where a sum is not finite
__global__ __launch_bounds__(kThreads) void ffn_parts_sum_kernel(const float *__restrict__ part, i64 M, i64 D, i64 ld,
                                                                 int splits, int tiles_d, float *__restrict__ dX,
                                                                 Whole whole)
{
    __shared__ float lds[kAnyFloats];
    const i64 r0 = (i64)(blockIdx.x / tiles_d) * kSumRows, c0 = (i64)(blockIdx.x % tiles_d) * kTN;
    const i64 m = r0 + threadIdx.x / (kTN / 4), d = c0 + threadIdx.x % (kTN / 4) * 4;
    const bool in = m < M && d < ld;
    const float *p = part + (in ? m * ld + d : 0);
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < splits; k += 8) {
        float4 q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            q[j] = k + j < splits ? *reinterpret_cast<const float4 *>(p + (i64)(k + j) * M * ld)
                                  : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[0] += q[j].x;
            v[1] += q[j].y;
            v[2] += q[j].z;
            v[3] += q[j].w;
        }
    }
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) bad |= in && d + j < D && !split::finite_f32(v[j]);
    if (__syncthreads_or(bad)) {
        any_dx_tile<kThreads>(whole.a, whole.b, whole.wg, whole.wu, r0 + kSumRows < M ? r0 + kSumRows : M, D, whole.K, r0,
                              c0, dX, lds);
        return;
    }
    if (!in) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (d + j < D) dX[m * D + d + j] = v[j] * split::kUnscale;
}

// ---------------------------------------------------------------------------
// the parts
// ---------------------------------------------------------------------------
// Arrays to split: P [rows][cols] as the kilobytes of its parts at O (Parts,
// or, by_cols, as W of ffn_parts_dx_kernel), zeros past rows and cols.  One
// launch for all of a call's, a wave per kilobyte of values' worth (the three
// parts of 64 pieces of eight), first[k] the first of array k, of at most
// kSplitBlocks workgroups.
struct Splits {
    int count;
    const float *P[4];
    char *O[4];
    i64 rows[4], cols[4], stages[4], first[5];
    int by_cols[4];
};

__global__ __launch_bounds__(256) void ffn_split_kernel(Splits s)
{
    const int lane = threadIdx.x & 63;
    const i64 wave = (i64)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (i64 i = wave; i < s.first[s.count]; i += (i64)gridDim.x * 4) {
        int k = 0;
        while (k + 1 < s.count && i >= s.first[k + 1]) ++k;
        const i64 rows = s.rows[k], cols = s.cols[k], t = i - s.first[k];
        i64 r, c, at, step;               // the piece's place in P; the first part's kilobyte and the way to the next
        if (s.by_cols[k]) {
            const i64 g = t % kWLoads, cs = t / kWLoads, cb = cs / s.stages[k], st = cs - cb * s.stages[k];
            const int row = lane / 16;
            r = st * kBK + g * kWRpi + row;
            c = cb * kCols + 8 * ((lane % 16) ^ (4 * (row & 3)));
            at = cs * kPlanes * kWLoads + g;
            step = kWLoads;
        } else {
            const i64 group = t / s.stages[k], st = t - group * s.stages[k];
            const int row = lane / (64 / kRpi);
            r = group * kRpi + row;
            c = st * kBK + 8 * piece_of(row, lane % (64 / kRpi));
            at = t * kPlanes;
            step = 1;
        }
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
        for (int q = 0; q < 4; ++q) split::split2(x[2 * q], x[2 * q + 1], w[0][q], w[1][q], w[2][q]);
#pragma unroll
        for (int n = 0; n < 3; ++n)
            *reinterpret_cast<uint4 *>(s.O[k] + (at + n * step) * 1024 + 16 * lane) =
                make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]);
    }
}

i64 stages_of(i64 features) { return ceil_div(features, kBK); }

// kilobytes of one part of [rows][features], and of [features][cols] by columns
i64 row_parts(i64 rows, i64 features) { return ceil_div(rows, kRpi) * stages_of(features); }
i64 col_parts(i64 features, i64 cols) { return ceil_div(cols, kCols) * stages_of(features) * kWLoads; }

// Adds P's split at ws, which is moved on; returns where.
char *add_split(Splits &s, const float *P, i64 rows, i64 cols, bool by_cols, char *&ws)
{
    const int k = s.count++;
    const i64 n = by_cols ? col_parts(rows, cols) : row_parts(rows, cols);
    s.P[k] = P;
    s.O[k] = ws;
    s.rows[k] = rows;
    s.cols[k] = cols;
    s.stages[k] = stages_of(by_cols ? rows : cols);
    s.by_cols[k] = by_cols;
    s.first[k + 1] = s.first[k] + n;
    ws += kPlanes * 1024 * n;
    return s.O[k];
}

Parts add_rows(Splits &s, const float *P, i64 rows, i64 cols, char *&ws)
{
    const char *p = add_split(s, P, rows, cols, false, ws);
    return Parts{p, ceil_div(rows, kRpi), stages_of(cols)};
}

void split_arrays(const Splits &s, hipStream_t stream)
{
    const i64 blocks = ceil_div(s.first[s.count], 4);
    ffn_split_kernel<<<(unsigned)(blocks < kSplitBlocks ? blocks : kSplitBlocks), 256, 0, stream>>>(s);
}

// Splits of the features by the time they take: a stage at 0.55 us while most
// workgroups have a CU to themselves, at 1.39 us per round of two per CU, the
// first loads and last stores, and the partial tiles written and read.
// 512 x 2752 -> 1024 (32 tiles), the whole call: 183 us in one split, 68 in
// four, 60 in six and in eight, 71 in sixteen; 4096 x 2752 -> 1024 (256 tiles)
// 304 in one, 309 in two, 334 in eight.
int dx_splits(i64 M, i64 D, i64 F)
{
    const i64 stages = 2 * stages_of(F), tiles = ceil_div(M, DxTile::BM) * ceil_div(D, DxTile::BD);
    double best = 1e30;
    int splits = 1;
    for (int s = 1; s <= 16 && s <= stages / 4 + 1; ++s) {
        const double n = (double)tiles * s, stage = n <= 192 ? 0.55 : n <= 512 ? 0.21 + 0.0023 * n : 1.39 * n / 512;
        const double t = stage * (double)ceil_div(stages, s) + 3.0 * n / 512 +
                         (s > 1 ? 4.0 + 8.0 * s * (double)M * (double)D / 4.5e6 : 0.0);
        if (t < best) {
            best = t;
            splits = s;
        }
    }
    return splits;
}

}  // namespace

size_t ffn_parts_forward_workspace(i64 M, i64 K, i64 F)
{
    return kPlanes * 1024 * (size_t)(row_parts(M, K) + 2 * row_parts(F, K));
}

void ffn_parts_forward(const float *X, const float *Wg, const float *Wu, i64 M, i64 K, i64 F, dp_act act, float *H,
                       float *G, float *U, void *ws, hipStream_t stream)
{
    char *w = (char *)ws;
    Splits s = {};
    const Parts x = add_rows(s, X, M, K, w), g = add_rows(s, Wg, F, K, w), u = add_rows(s, Wu, F, K, w);
    split_arrays(s, stream);
    const Whole whole = {X, nullptr, Wg, Wu, K};
    const int tm = (int)ceil_div(M, Tile::BM), tf = (int)ceil_div(F, Tile::BF);
    const int vec = F % 4 == 0 && aligned(H, 16) && aligned(G, 16) && aligned(U, 16);
    const unsigned grid = (unsigned)((i64)tm * tf);
    if (act == DP_ACT_SILU)
        ffn_parts_forward_kernel<Tile, DP_ACT_SILU><<<grid, kThreads, 0, stream>>>(x, g, u, M, F, tm, tf, H, G, U, vec,
                                                                                  whole);
    else
        ffn_parts_forward_kernel<Tile, DP_ACT_GELU_TANH><<<grid, kThreads, 0, stream>>>(x, g, u, M, F, tm, tf, H, G, U,
                                                                                       vec, whole);
}

size_t ffn_parts_dx_workspace(i64 M, i64 D, i64 F)
{
    const int splits = dx_splits(M, D, F);
    const size_t part = splits > 1 ? sizeof(float) * (size_t)splits * (size_t)(M * padded(D)) : 0;
    return kPlanes * 1024 * (size_t)(2 * row_parts(M, F) + 2 * col_parts(F, D)) + part;
}

void ffn_parts_dx(const float *BG, const float *BU, const float *Wg, const float *Wu, i64 M, i64 D, i64 F, float *dX,
                  void *ws, hipStream_t stream)
{
    const i64 ldw = padded(D);
    const int splits = dx_splits(M, D, F);
    char *w = (char *)ws;
    Splits s = {};
    const Parts g = add_rows(s, BG, M, F, w), u = add_rows(s, BU, M, F, w);
    const char *W = add_split(s, Wg, F, D, true, w);
    add_split(s, Wu, F, D, true, w);                         // behind Wg's
    float *part = (float *)w;
    split_arrays(s, stream);
    const Whole whole = {BG, BU, Wg, Wu, F};
    const int tm = (int)ceil_div(M, DxTile::BM), td = (int)ceil_div(D, DxTile::BD);
    const int vec = D % 4 == 0 && aligned(dX, 16);
    const unsigned grid = (unsigned)((i64)tm * td * splits);
    if (splits == 1) {
        ffn_parts_dx_kernel<false><<<grid, kThreads, 0, stream>>>(g, u, W, M, D, ldw, tm, td, 1, dX, nullptr, vec, whole);
        return;
    }
    ffn_parts_dx_kernel<true><<<grid, kThreads, 0, stream>>>(g, u, W, M, D, ldw, tm, td, splits, dX, part, vec, whole);
    // (several splits only of up to 512 tiles: a grid of at most 8192 workgroups)
    const i64 cols = ceil_div(D, kTN);
    ffn_parts_sum_kernel<<<(unsigned)(ceil_div(M, kSumRows) * cols), kThreads, 0, stream>>>(part, M, D, ldw, splits,
                                                                                           (int)cols, dX, whole);
}

}  // namespace dpg
