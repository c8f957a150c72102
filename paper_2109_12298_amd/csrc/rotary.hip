// Rotary positions: pair j of a head turned by the angle pos * freq[j].
//
// Bound by its bytes: every value is read and written once.  A workgroup takes
// some positions, forms each (position, pair)'s sine and cosine once, in LDS,
// and turns all heads by them; a thread keeps its pairs and has the loads of
// kAhead heads in flight.  An angle is pos * freq / (2 pi) in 64 bits less the
// nearest whole number of turns, then sine and cosine of what is left (within
// half a turn) in fp32: the quotient's error is at most 3 * 2^-53 of the angle
// (the product, the constant and the quotient, each rounded), so that positions of
// 2^20 and more keep all of fp32's bits.
//
// 4 x 4096 positions, 40 heads of 128 out of 56, three axes, bf16: 63 us, 5.3 TB/s
// (a copy's rate is 4.9).  One position: 3 us, the angles' 64-bit arithmetic and
// one trip to memory.
#include "common.hpp"

namespace dpg {
namespace {

constexpr int kThreads = 256;           // aimed at; a wide head's slots may take more
constexpr int kMaxThreads = 1024;
constexpr int kMaxD = 1024;
constexpr int kAhead = 4;
constexpr int kMaxAxes = 4;
constexpr i64 kMaxGrid = i64(1) << 21;

struct Axes {
    int end[kMaxAxes];                  // first pair after each axis' section
    int count;
};

// N consecutive elements, as loaded (one 16-byte piece at the most); two of
// them in the layout of adjacent pairs may lie at an odd place
template <typename T, int N, int ALIGN = N>
struct alignas(sizeof(T) * ALIGN) Pack {
    T v[N];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ void from_f32(float x, float &y) { y = x; }
__device__ __forceinline__ void from_f32(float x, uint16_t &y)
{
    const __bf16 b = (__bf16)x;
    y = __builtin_bit_cast(uint16_t, b);
}

// A slot is what a thread has of a head: NP pairs (from two places of the head
// in the layout of halves, 2 NP consecutive values in the other), or W
// consecutive values behind the pairs, copied.  `heads` heads side by side;
// `at_once` positions side by side, `per_block` in all.
template <typename T, bool HALVES, int NP, int W>
__global__ __launch_bounds__(kMaxThreads) void rotary_kernel(const T *X, i64 M, int H, int D, int P, i64 ldx,
                                                             const int64_t *__restrict__ pos, Axes ax,
                                                             const double *__restrict__ freq, float sign, T *Y, i64 ldy,
                                                             int slots, int heads, int at_once, int per_block)
{
    constexpr int N = HALVES ? NP : 2 * NP;             // consecutive values
    typedef Pack<T, N, (W < N ? W : N)> Piece;
    extern __shared__ float2 turn[];                    // [per_block][P]: cosine, sine
    const int per_pos = slots * heads;
    const int at = (int)threadIdx.x / per_pos, in = (int)threadIdx.x - at * per_pos;
    const int h0 = in / slots, slot = in - h0 * slots;
    const int turning = P / NP;
    for (i64 m0 = (i64)blockIdx.x * per_block; m0 < M; m0 += (i64)gridDim.x * per_block) {
        const int count = (int)(M - m0 < per_block ? M - m0 : per_block);
        for (int e = threadIdx.x; e < count * P; e += blockDim.x) {
            const int k = e / P, j = e - k * P;
            int a = 0;
            while (a + 1 < ax.count && j >= ax.end[a]) ++a;
            const double turns = (double)pos[a * M + m0 + k] * freq[j] * 0.15915494309189535;
            float s, c;
            sincospif(2.0f * (float)(turns - __builtin_rint(turns)), &s, &c);
            turn[e] = make_float2(c, sign * s);
        }
        __syncthreads();
        if (at < at_once)
            for (int k = at; k < count; k += at_once) {
                const T *x = X + (m0 + k) * ldx;
                T *y = Y + (m0 + k) * ldy;
                if (slot >= turning) {
                    const int d = 2 * P + (slot - turning) * W;
                    for (int h = h0; h < H; h += heads)
                        *reinterpret_cast<Pack<T, W> *>(y + h * D + d) = *reinterpret_cast<const Pack<T, W> *>(x + h * D + d);
                    continue;
                }
                float c[NP], s[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const float2 t = turn[k * P + slot * NP + i];
                    c[i] = t.x;
                    s[i] = t.y;
                }
                const int d = slot * N;
                for (int hb = h0; hb < H; hb += kAhead * heads) {
                    Piece u[kAhead], v[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int h = hb + i * heads < H ? hb + i * heads : hb;        // past the end: read again, not stored
                        u[i] = *reinterpret_cast<const Piece *>(x + h * D + d);
                        if constexpr (HALVES) v[i] = *reinterpret_cast<const Piece *>(x + h * D + d + P);
                    }
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int h = hb + i * heads;
                        if (h >= H) break;
                        Piece a, b;
#pragma unroll
                        for (int e = 0; e < NP; ++e) {
                            const float f = to_f32(HALVES ? u[i].v[e] : u[i].v[2 * e]);
                            const float g = to_f32(HALVES ? v[i].v[e] : u[i].v[2 * e + 1]);
                            from_f32(f * c[e] - g * s[e], HALVES ? a.v[e] : a.v[2 * e]);
                            from_f32(g * c[e] + f * s[e], HALVES ? b.v[e] : a.v[2 * e + 1]);
                        }
                        *reinterpret_cast<Piece *>(y + h * D + d) = a;
                        if constexpr (HALVES) *reinterpret_cast<Piece *>(y + h * D + d + P) = b;
                    }
                }
            }
        __syncthreads();
    }
}

struct Call {
    const void *X;
    i64 M, H, D, P, ldx;
    const int64_t *pos;
    Axes ax;
    const double *freq;
    float sign;
    void *Y;
    i64 ldy;
    hipStream_t stream;
};

template <typename T, bool HALVES, int NP, int W>
dp_status launch(const Call &c)
{
    const i64 slots = c.P / NP + (c.X == c.Y ? 0 : (c.D - 2 * c.P) / W);
    if (slots == 0) return DP_OK;                        // in place, nothing to turn
    // heads side by side: as many as a workgroup holds, evenly over its passes
    const i64 fit = slots < kThreads ? kThreads / slots : 1;
    const i64 heads = ceil_div(c.H, ceil_div(c.H, fit));
    const i64 per_pos = slots * heads;
    const i64 at_once = per_pos < kThreads ? kThreads / per_pos : 1;
    // four rounds of positions, so that all threads form angles, where that leaves workgroups enough
    const i64 rounds = ceil_div(c.M, 4 * at_once) >= 1024 && 4 * at_once * c.P <= 1024 ? 4 : 1, per_block = at_once * rounds;
    i64 grid = ceil_div(c.M, per_block);
    if (grid > kMaxGrid) grid = kMaxGrid;
    const unsigned threads = (unsigned)(ceil_div(per_pos * at_once, kWave) * kWave);
    rotary_kernel<T, HALVES, NP, W><<<(unsigned)grid, threads, sizeof(float2) * per_block * c.P, c.stream>>>(
        (const T *)c.X, c.M, (int)c.H, (int)c.D, (int)c.P, c.ldx, c.pos, c.ax, c.freq, c.sign, (T *)c.Y, c.ldy, (int)slots,
        (int)heads, (int)at_once, (int)per_block);
    return launch_status();
}

// the widest pieces that every head's start and every section allow
template <typename T>
dp_status by_width(const Call &c, dp_rotary_layout layout)
{
    const auto fits = [&](i64 n) {
        return c.D % n == 0 && c.ldx % n == 0 && c.ldy % n == 0 && aligned(c.X, n * sizeof(T)) && aligned(c.Y, n * sizeof(T)) &&
               (layout == DP_ROTARY_HALVES ? c.P : 2 * c.P) % n == 0;
    };
    constexpr int N = 16 / sizeof(T);
    if (layout == DP_ROTARY_HALVES) {
        if (fits(N)) return launch<T, true, N, N>(c);
        if (fits(2)) return launch<T, true, 2, 2>(c);
        return launch<T, true, 1, 1>(c);
    }
    if (fits(N)) return launch<T, false, N / 2, N>(c);
    return launch<T, false, 1, 1>(c);
}

}  // namespace
}  // namespace dpg

using namespace dpg;

extern "C" dp_status dp_rotary(const void *X, dp_dtype dt, int64_t N, int64_t T, int64_t H, int64_t D, int64_t ldx,
                               const int64_t *pos, const int64_t *sections, int32_t axes, const double *freq,
                               dp_rotary_layout layout, int32_t inverse, void *Y, int64_t ldy, hipStream_t stream)
{
    DPG_REQUIRE(dtype_ok(dt), DP_EDTYPE);
    DPG_REQUIRE(N >= 0 && T >= 0 && H >= 1 && D >= 1 && axes >= 1 && axes <= kMaxAxes, DP_EINVAL);
    DPG_REQUIRE(layout == DP_ROTARY_HALVES || layout == DP_ROTARY_ADJACENT, DP_EINVAL);
    DPG_REQUIRE(N < (i64(1) << 31) && T < (i64(1) << 31) && N * T < (i64(1) << 31), DP_EUNSUPPORTED);
    DPG_REQUIRE(D <= kMaxD && H < (i64(1) << 20), DP_EUNSUPPORTED);
    DPG_REQUIRE(ldx >= H * D && ldy >= H * D, DP_EINVAL);
    DPG_REQUIRE(ldx < (i64(1) << 31) && ldy < (i64(1) << 31), DP_EUNSUPPORTED);
    DPG_REQUIRE(sections != nullptr, DP_EINVAL);
    Call c = {X, N * T, H, D, 0, ldx, pos, {}, freq, inverse != 0 ? -1.0f : 1.0f, Y, ldy, stream};
    c.ax.count = axes;
    for (int a = 0; a < axes; ++a) {
        DPG_REQUIRE(sections[a] >= 0 && sections[a] <= D, DP_EINVAL);
        c.P += sections[a];
        c.ax.end[a] = (int)c.P;
    }
    DPG_REQUIRE(2 * c.P <= D, DP_EINVAL);
    if (c.M == 0) return DP_OK;
    DPG_REQUIRE(X != nullptr && Y != nullptr && pos != nullptr && (freq != nullptr || c.P == 0), DP_EINVAL);
    DPG_REQUIRE(aligned(X, dtype_bytes(dt)) && aligned(Y, dtype_bytes(dt)) && aligned(pos, 8) && aligned(freq, 8), DP_EINVAL);
    DPG_REQUIRE(X != Y || ldx == ldy, DP_EINVAL);
    return dt == DP_F32 ? by_width<float>(c, layout) : by_width<uint16_t>(c, layout);
}
