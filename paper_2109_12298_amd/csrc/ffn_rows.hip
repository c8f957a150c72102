// Gated feed-forward block over few rows (a decoding step's single token up
// to 64 rows): bound by reading Wg and Wu once.
//
// A workgroup takes 16 features of Wg and Wu and all rows of X; its waves
// split K in units of 128 bytes of a row, unit by unit in turn, so that the
// workgroup reads each weight row front to back.  Weights go straight from
// memory to registers in the operand layout of v_mfma_f32_16x16x32_bf16 (or
// v_mfma_f32_16x16x4_f32): lane l holds 16 bytes of feature l % 16; the
// matrix unit's columns are the rows of X (rows past M repeat the last one
// and are not stored).  X comes from the caches.  The waves' sums meet in LDS,
// added in wave order, where G, U and H are formed.
//
// For fp32 a lane's four consecutive values k .. k + 3 feed four products,
// whose k index runs over the lane groups: any order of K serves, as long as
// both operands use the same.
#include "ffn_rows.hpp"

#include "gated_ffn.hpp"

namespace dpg {
namespace {

using namespace ffn;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kFT = 16;                   // features per workgroup

template <typename T>
struct Piece {                            // a lane's share of one step: 16 bytes of a row
    static constexpr int N = 16 / sizeof(T);
    static constexpr int STEP = 4 * N;    // columns of a step (four lane groups); two steps are a unit of 128 bytes
    alignas(16) T v[N];
};

// columns k .. k + N - 1 of the row at p, zeros at and past K
template <typename T, bool VEC>
__device__ __forceinline__ Piece<T> load_cut(const T *p, i64 k, i64 K)
{
    constexpr int N = Piece<T>::N;
    Piece<T> r;
    if constexpr (VEC) {                  // K is a multiple of N: all in or all out
        r = *reinterpret_cast<const Piece<T> *>(p + (k < K ? k : 0));
#pragma unroll
        for (int j = 0; j < N; ++j) r.v[j] = k < K ? r.v[j] : T(0);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) r.v[j] = k + j < K ? p[k + j] : T(0);
    }
    return r;
}

template <typename T, bool VEC>
__device__ __forceinline__ Piece<T> load_full(const T *p, i64 k)
{
    Piece<T> r;
    if constexpr (VEC) {
        r = *reinterpret_cast<const Piece<T> *>(p + k);
    } else {
#pragma unroll
        for (int j = 0; j < Piece<T>::N; ++j) r.v[j] = p[k + j];
    }
    return r;
}

__device__ __forceinline__ void mma(const Piece<uint16_t> &a, const Piece<uint16_t> &b, f32x4_t &c)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a.v), __builtin_bit_cast(bf16x8_t, b.v), c,
                                                0, 0, 0);
}
__device__ __forceinline__ void mma(const Piece<float> &a, const Piece<float> &b, f32x4_t &c)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
}

template <int MB>
constexpr int max_waves() { return MB <= 2 ? 16 : 8; }            // 64 KB of LDS for the sums

// MB: blocks of 16 rows of X; UNITS: units whose loads a wave has in flight
template <typename T, int ACT, int MB, int UNITS, bool VEC>
__global__ __launch_bounds__(64 * max_waves<MB>()) void ffn_rows_kernel(const T *__restrict__ X,
                                                                        const T *__restrict__ Wg,
                                                                        const T *__restrict__ Wu, int M, i64 K, i64 F,
                                                                        T *__restrict__ H, T *__restrict__ G,
                                                                        T *__restrict__ U)
{
    constexpr int STEP = Piece<T>::STEP, UNIT = 2 * STEP, N = Piece<T>::N;
    extern __shared__ f32x4_t red[];      // [waves][2][MB][64]
    const int lane = threadIdx.x & 63, waves = (int)blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const i64 f0 = (i64)blockIdx.x * kFT;
    const int li = lane & 15, k0 = lane / 16 * N;
    const i64 f = f0 + li < F ? f0 + li : F - 1;
    const T *wg = Wg + f * K, *wu = Wu + f * K;
    const T *x[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) x[b] = X + (i64)(16 * b + li < M ? 16 * b + li : M - 1) * K;

    f32x4_t ag[MB], au[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) ag[b] = au[b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const i64 whole = K / UNIT;           // whole units; one cut unit may follow
    i64 u = wave;
    for (; u + (i64)(UNITS - 1) * waves < whole; u += (i64)UNITS * waves) {
        Piece<T> pg[UNITS][2], pu[UNITS][2], px[UNITS][2][MB];
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const i64 k = (u + (i64)i * waves) * UNIT + s * STEP + k0;
                pg[i][s] = load_full<T, VEC>(wg, k);
                pu[i][s] = load_full<T, VEC>(wu, k);
#pragma unroll
                for (int b = 0; b < MB; ++b) px[i][s][b] = load_full<T, VEC>(x[b], k);
            }
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    mma(pg[i][s], px[i][s][b], ag[b]);
                    mma(pu[i][s], px[i][s][b], au[b]);
                }
    }
    for (; u * UNIT < K; u += waves) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const i64 k = u * UNIT + s * STEP + k0;
            const Piece<T> pg = load_cut<T, VEC>(wg, k, K), pu = load_cut<T, VEC>(wu, k, K);
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                const Piece<T> px = load_cut<T, VEC>(x[b], k, K);
                mma(pg, px, ag[b]);
                mma(pu, px, au[b]);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        red[(wave * 2 * MB + b) * 64 + lane] = ag[b];
        red[(wave * 2 * MB + MB + b) * 64 + lane] = au[b];
    }
    __syncthreads();
    // register r of lane l: feature 4 (l / 16) + r, row l % 16
    const float *v = reinterpret_cast<const float *>(red);
    for (int e = threadIdx.x; e < MB * 256; e += (int)blockDim.x) {
        // consecutive threads take consecutive features of a row
        const int b = e >> 8, i = (e & 255) >> 4, fe = e & 15;
        const int row = 16 * b + i, src = (b * 64 + (fe >> 2) * 16 + i) * 4 + (fe & 3);
        float g = 0.0f, uu = 0.0f;
        for (int w = 0; w < waves; ++w) {
            g += v[w * 2 * MB * 256 + src];
            uu += v[w * 2 * MB * 256 + MB * 256 + src];
        }
        if (row >= M || f0 + fe >= F) continue;
        const i64 o = (i64)row * F + f0 + fe;
        store_elem(H + o, act_for<ACT, T>(g) * uu);
        if (G != nullptr) {
            store_elem(G + o, g);
            store_elem(U + o, uu);
        }
    }
}

template <typename T, int ACT, int MB, int UNITS>
void launch(const void *X, const void *Wg, const void *Wu, i64 M, i64 K, i64 F, void *H, void *G, void *U,
            hipStream_t stream)
{
    const i64 groups = ceil_div(F, kFT), units = ceil_div(K, 2 * Piece<T>::STEP);
    // four waves, or more where the features alone give too few waves to fill the GPU and K has units for them
    int waves = 4;
    while (waves < max_waves<MB>() && groups * waves < 2048 && units >= 2 * waves * UNITS) waves *= 2;
    const size_t lds = (size_t)waves * 2 * MB * 64 * sizeof(f32x4_t);
    const bool vec = K % Piece<T>::N == 0 && aligned(X, 16) && aligned(Wg, 16) && aligned(Wu, 16);
    const auto go = [&](auto kernel) {
        kernel<<<(unsigned)groups, 64 * waves, lds, stream>>>((const T *)X, (const T *)Wg, (const T *)Wu, (int)M, K, F,
                                                              (T *)H, (T *)G, (T *)U);
    };
    // (aligned bf16 rows above kFfnRowsBf16 go to the tiles, but for d_in from 2^21 on: single loads do for those)
    constexpr bool VEC = sizeof(T) == 4 || MB == 1;
    if (VEC && vec) go(ffn_rows_kernel<T, ACT, MB, UNITS, VEC>);
    else go(ffn_rows_kernel<T, ACT, MB, UNITS, false>);
}

template <typename T, int ACT>
void by_rows(const void *X, const void *Wg, const void *Wu, i64 M, i64 K, i64 F, void *H, void *G, void *U,
             hipStream_t stream)
{
    // units in flight, measured at 4096 -> 11008 alone and taken for all sizes: one row bf16 37.8 us with 2, 38.0 with 1,
    // 41 with 4; fp32 32 rows 104 us with 1, 119 with 2; 64 rows 165 with 3, 179 with 1
    if (M <= 16) launch<T, ACT, 1, 2>(X, Wg, Wu, M, K, F, H, G, U, stream);
    else if (M <= 32) launch<T, ACT, 2, 1>(X, Wg, Wu, M, K, F, H, G, U, stream);
    else launch<T, ACT, 4, 3>(X, Wg, Wu, M, K, F, H, G, U, stream);
}

template <typename T>
void by_act(const void *X, const void *Wg, const void *Wu, i64 M, i64 K, i64 F, dp_act act, void *H, void *G, void *U,
            hipStream_t stream)
{
    if (act == DP_ACT_SILU) by_rows<T, DP_ACT_SILU>(X, Wg, Wu, M, K, F, H, G, U, stream);
    else by_rows<T, DP_ACT_GELU_TANH>(X, Wg, Wu, M, K, F, H, G, U, stream);
}

// ---------------------------------------------------------------------------
// dX = BG Wg + BU Wu in fp32 over few rows: a workgroup takes 128 columns and a
// run of the features of both products, its waves every fourth group of eight
// features.  Weights go straight to the operands of v_mfma_f32_32x32x2_f32: a
// lane loads 16 bytes of a weight row (columns 4 j .. 4 j + 3, j = lane % 32),
// which feed four products with the same column index j, and features are
// dealt to the k index so that a lane's share of BG is 16 consecutive bytes.
// The waves' sums are added in LDS in wave order, the workgroups' from the
// workspace in order.  Weights are read once, past the caches (one row, 11008 ->
// 4096: the call 86 us, 82 so, 360 MB; 11008 -> 4096 bf16 in the tiles of
// ffn_bf16.hip likewise 41 and 37 us).
// ---------------------------------------------------------------------------
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kDxCols = 128, kDxWaves = 4, kDxGroup = 8;

// four consecutive values of the row at p from index k on, zeros from `end`
// on; STREAM: past the caches
template <bool VEC, bool STREAM = false>
__device__ __forceinline__ float4 load4(const float *p, i64 k, i64 end)
{
    if constexpr (VEC) {                  // end is a multiple of 4, p 16-byte aligned
        const float *q = p + (k < end ? k : 0);
        const float4 v = STREAM ? load_stream4(q) : *reinterpret_cast<const float4 *>(q);
        return k < end ? v : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    } else {
        return make_float4(k < end ? p[k] : 0.0f, k + 1 < end ? p[k + 1] : 0.0f, k + 2 < end ? p[k + 2] : 0.0f,
                           k + 3 < end ? p[k + 3] : 0.0f);
    }
}

template <int MB, bool VEC>
__global__ __launch_bounds__(64 * kDxWaves) void ffn_dx_rows_kernel(const float *__restrict__ BG,
                                                                    const float *__restrict__ BU,
                                                                    const float *__restrict__ Wg,
                                                                    const float *__restrict__ Wu, int M, i64 D, i64 F,
                                                                    int colblocks, int splits, float *__restrict__ out)
{
    constexpr int UNROLL = MB == 1 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) float red[MB * 4 * 1024];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 31, lk = lane >> 5;
    const int cb = (int)blockIdx.x % colblocks, split = (int)blockIdx.x / colblocks;
    const i64 d = (i64)cb * kDxCols + 4 * li;
    f32x16_t acc[MB][4];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][i][r] = 0.0f;

    // groups of eight features of BG, then of BU
    const i64 half = (F + kDxGroup - 1) / kDxGroup;
    const i64 g0 = (i64)split * 2 * half / splits, g1 = (i64)(split + 1) * 2 * half / splits;
    for (i64 gb = g0 + wave; gb < g1; gb += UNROLL * kDxWaves) {
        float4 w[UNROLL][4], a[UNROLL][MB];
#pragma unroll
        for (int n = 0; n < UNROLL; ++n) {
            const i64 g = gb + n * kDxWaves;
            const bool u = g >= half;
            // features f .. f + 3 of this lane; past the end (of the run, too) zeros on both sides
            const i64 f = (u ? g - half : g) * kDxGroup + 4 * lk, end = g < g1 ? F : 0;
            const float *W = u ? Wu : Wg, *B = u ? BU : BG;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bool in = f + s < end;
                const float4 v = load4<VEC, true>(W + (in ? f + s : 0) * D, d, D);
                w[n][s] = in ? v : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int b = 0; b < MB; ++b) a[n][b] = load4<VEC>(B + (i64)(32 * b + li < M ? 32 * b + li : M - 1) * F, f, end);
        }
#pragma unroll
        for (int n = 0; n < UNROLL; ++n)
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    const float x = s == 0 ? a[n][b].x : s == 1 ? a[n][b].y : s == 2 ? a[n][b].z : a[n][b].w;
                    acc[b][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[n][s].x, x, acc[b][0], 0, 0, 0);
                    acc[b][1] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[n][s].y, x, acc[b][1], 0, 0, 0);
                    acc[b][2] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[n][s].z, x, acc[b][2], 0, 0, 0);
                    acc[b][3] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[n][s].w, x, acc[b][3], 0, 0, 0);
                }
    }
    // acc[b][i][r] of lane l: row 32 b + l % 32, column 4 j + i, j = 8 (r / 4) + 4 (l / 32) + r % 4
    for (int w = 0; w < kDxWaves; ++w) {
        if (wave == w) {
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = 8 * (r >> 2) + 4 * lk + (r & 3);
                    float4 *p = reinterpret_cast<float4 *>(red) + (32 * b + li) * 32 + (j ^ (li & 31));
                    float4 v = make_float4(acc[b][0][r], acc[b][1][r], acc[b][2][r], acc[b][3][r]);
                    if (w > 0) {
                        const float4 o = *p;
                        v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
                    }
                    *p = v;
                }
        }
        __syncthreads();
    }
    float *O = out + (i64)split * M * D;
    for (int e = threadIdx.x; e < 32 * MB * 32; e += 64 * kDxWaves) {
        const int row = e >> 5, j = e & 31;
        const i64 c = (i64)cb * kDxCols + 4 * j;
        if (row >= M || c >= D) continue;
        const float4 v = reinterpret_cast<const float4 *>(red)[row * 32 + (j ^ (row & 31))];
        const float x[4] = {v.x, v.y, v.z, v.w};
        if (D % 4 == 0 && (reinterpret_cast<uintptr_t>(O) & 15) == 0) {
            *reinterpret_cast<float4 *>(O + row * D + c) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < D) O[row * D + c + i] = x[i];
        }
    }
}

// out = the splits' sums, in split order
__global__ __launch_bounds__(256) void ffn_dx_rows_sum_kernel(const float *__restrict__ part, i64 n, int splits,
                                                              float *__restrict__ out)
{
    for (i64 i = (i64)blockIdx.x * 256 + threadIdx.x; i < n; i += (i64)gridDim.x * 256)
        out[i] = ordered_sum(part + i, n, splits);
}

// Runs of features by the time they take: 32 features at 0.75 us (1.35 over 32
// rows) per round of 256 workgroups; more than one run takes one more launch
// and writes and reads partial sums.  64 x 4096 -> 4096: 182 us in two runs, 59
// in eight, 81 in twelve, 69 in sixteen; one row of 100 -> 256: 12.5 in one,
// 14.3 in two.
int dx_rows_splits(i64 M, i64 D, i64 F)
{
    const i64 units = ceil_div(2 * ceil_div(F, kDxGroup), kDxWaves), cols = ceil_div(D, kDxCols);
    const double unit = M <= 32 ? 0.75 : 1.35;
    double best = unit * (double)(units * ceil_div(cols, 256));
    int splits = 1;
    for (int s = 2; s <= 64 && 2 * s <= units; ++s) {
        const double t = unit * (double)(ceil_div(units, s) * ceil_div(cols * s, 256)) + 7.0 +
                         16.0 * s * (double)M * (double)D / 4.5e6;
        if (t < best) {
            best = t;
            splits = s;
        }
    }
    return splits;
}

}  // namespace

void ffn_rows_forward(const void *X, const void *Wg, const void *Wu, dp_dtype dt, i64 M, i64 K, i64 F, dp_act act,
                      void *H, void *G, void *U, hipStream_t stream)
{
    if (dt == DP_F32) by_act<float>(X, Wg, Wu, M, K, F, act, H, G, U, stream);
    else by_act<uint16_t>(X, Wg, Wu, M, K, F, act, H, G, U, stream);
}

size_t ffn_rows_dx_workspace(i64 M, i64 D, i64 F)
{
    const int splits = dx_rows_splits(M, D, F);
    return splits > 1 ? sizeof(float) * (size_t)splits * (size_t)(M * D) : 0;
}

void ffn_rows_dx(const float *BG, const float *BU, const float *Wg, const float *Wu, i64 M, i64 D, i64 F, float *dX,
                 void *ws, hipStream_t stream)
{
    const int splits = dx_rows_splits(M, D, F), cb = (int)ceil_div(D, kDxCols);
    const bool vec = D % 4 == 0 && F % 4 == 0 && aligned(BG, 16) && aligned(BU, 16) && aligned(Wg, 16) && aligned(Wu, 16);
    float *out = splits > 1 ? (float *)ws : dX;
    const auto go = [&](auto kernel) {
        kernel<<<(unsigned)((i64)cb * splits), 64 * kDxWaves, 0, stream>>>(BG, BU, Wg, Wu, (int)M, D, F, cb, splits, out);
    };
    if (M <= 32) go(vec ? ffn_dx_rows_kernel<1, true> : ffn_dx_rows_kernel<1, false>);
    else go(vec ? ffn_dx_rows_kernel<2, true> : ffn_dx_rows_kernel<2, false>);
    if (splits > 1) {
        const i64 blocks = ceil_div(M * D, 256);
        ffn_dx_rows_sum_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, stream>>>(out, M * D, splits, dX);
    }
}

}  // namespace dpg
