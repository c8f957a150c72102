// Gated feed-forward block: both projections, the activation and the product
// in one kernel, and its backward pass.
//   forward:   G = X Wg^T, U = X Wu^T, H = act(G) * U
//   backward:  BG = dH * U * act'(G), BU = dH * act(G), dX = BG Wg + BU Wu
//
// The forward computes a tile of G and the same tile of U in one workgroup
// (each wave holds both accumulators of its positions and features), so that
// H is formed from fp32 values in registers; G and U are written only where a
// backward pass wants them.
#include "ffn_any.hpp"
#include "ffn_bf16.hpp"
#include "ffn_rows.hpp"

namespace dpg {
namespace {

using namespace ffn;

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------
// bf16 of any size and alignment (ffn_any.hpp): a workgroup per 64 x 64 tile.
// ---------------------------------------------------------------------------
template <int ACT>
__global__ __launch_bounds__(kThreads) void ffn_forward_any_kernel(const uint16_t *__restrict__ X,
                                                                   const uint16_t *__restrict__ Wg,
                                                                   const uint16_t *__restrict__ Wu, i64 M, i64 K, i64 F,
                                                                   i64 tiles_f, uint16_t *__restrict__ H,
                                                                   uint16_t *__restrict__ G, uint16_t *__restrict__ U)
{
    __shared__ float lds[kAnyFloats];
    const i64 b = xcd_swizzle(blockIdx.x, gridDim.x);
    any_forward_tile<kThreads, ACT>(X, Wg, Wu, M, K, F, b / tiles_f * kTM, b % tiles_f * kTN, H, G, U, lds);
}

__global__ __launch_bounds__(kThreads) void ffn_dx_any_kernel(const uint16_t *__restrict__ BG,
                                                              const uint16_t *__restrict__ BU,
                                                              const uint16_t *__restrict__ Wg,
                                                              const uint16_t *__restrict__ Wu, i64 M, i64 D, i64 F,
                                                              i64 tiles_d, uint16_t *__restrict__ dX)
{
    __shared__ float lds[kAnyFloats];
    const i64 b = xcd_swizzle(blockIdx.x, gridDim.x);
    any_dx_tile<kThreads>(BG, BU, Wg, Wu, M, D, F, b / tiles_d * kTM, b % tiles_d * kTN, dX, lds);
}

// ---------------------------------------------------------------------------
// The elementwise half of the backward pass: three arrays read, two written,
// 16 bytes per lane and array where their alignment allows.
// No __restrict__: BG and BU may be dH, G or U themselves (each element is
// read before it is written, by the same thread).
// ---------------------------------------------------------------------------
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};

template <typename T, int ACT, int VEC>
__global__ __launch_bounds__(kThreads) void ffn_backprops_kernel(const T *dH, const T *G, const T *U, i64 n, T *BG,
                                                                 T *BU)
{
    const i64 step = (i64)gridDim.x * kThreads * VEC;
    for (i64 i = ((i64)blockIdx.x * kThreads + threadIdx.x) * VEC; i < n; i += step) {
        if (VEC == 1 || i + VEC <= n) {
            const Pack<T, VEC> h = *reinterpret_cast<const Pack<T, VEC> *>(dH + i);
            const Pack<T, VEC> g = *reinterpret_cast<const Pack<T, VEC> *>(G + i);
            const Pack<T, VEC> u = *reinterpret_cast<const Pack<T, VEC> *>(U + i);
            Pack<T, VEC> bg, bu;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float a, s;
                act_and_slope<ACT>(load_elem<T>(g.v, j), a, s);
                const float d = load_elem<T>(h.v, j);
                store_elem(bg.v + j, d * load_elem<T>(u.v, j) * s);
                store_elem(bu.v + j, d * a);
            }
            *reinterpret_cast<Pack<T, VEC> *>(BG + i) = bg;
            *reinterpret_cast<Pack<T, VEC> *>(BU + i) = bu;
        } else {
            for (i64 e = i; e < n; ++e) {
                float a, s;
                act_and_slope<ACT>(load_elem<T>(G, e), a, s);
                const float d = load_elem<T>(dH, e), u = load_elem<T>(U, e);
                store_elem(BG + e, d * u * s);
                store_elem(BU + e, d * a);
            }
        }
    }
}

template <int ACT>
void forward_any(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, uint16_t *H, uint16_t *G,
                 uint16_t *U, hipStream_t stream)
{
    const i64 tiles_f = ceil_div(F, kTN);
    ffn_forward_any_kernel<ACT><<<(unsigned)(ceil_div(M, kTM) * tiles_f), kThreads, 0, stream>>>(X, Wg, Wu, M, K, F, tiles_f,
                                                                                                H, G, U);
}

template <typename T, int ACT>
void backprops(const void *dH, const void *G, const void *U, i64 n, void *BG, void *BU, hipStream_t stream)
{
    constexpr int VEC = 16 / sizeof(T);
    const bool vec = aligned(dH, 16) && aligned(G, 16) && aligned(U, 16) && aligned(BG, 16) && aligned(BU, 16);
    const i64 blocks = ceil_div(n, (i64)kThreads * (vec ? VEC : 1));
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
    if (vec)
        ffn_backprops_kernel<T, ACT, VEC><<<grid, kThreads, 0, stream>>>((const T *)dH, (const T *)G, (const T *)U, n,
                                                                        (T *)BG, (T *)BU);
    else
        ffn_backprops_kernel<T, ACT, 1><<<grid, kThreads, 0, stream>>>((const T *)dH, (const T *)G, (const T *)U, n,
                                                                      (T *)BG, (T *)BU);
}

void dx_any(const uint16_t *BG, const uint16_t *BU, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 D, i64 F,
            uint16_t *dX, hipStream_t stream)
{
    const i64 tiles_d = ceil_div(D, kTN);
    ffn_dx_any_kernel<<<(unsigned)(ceil_div(M, kTM) * tiles_d), kThreads, 0, stream>>>(BG, BU, Wg, Wu, M, D, F, tiles_d, dX);
}

dp_status check_sizes(i64 M, i64 D, i64 F)
{
    DPG_REQUIRE(M >= 0 && D >= 1 && F >= 1, DP_EINVAL);
    // a grid holds fewer than 2^32 threads: 256 per 64 x 64 values, or per 16 features
    const i64 top = i64(1) << 27, most = i64(1) << 35;
    DPG_REQUIRE(M < top && D < top && F < top, DP_EUNSUPPORTED);
    DPG_REQUIRE(M * D < most && M * F < most && D * F < most, DP_EUNSUPPORTED);
    DPG_REQUIRE(ceil_div(M, kTM) * ceil_div(F > D ? F : D, kTN) < (i64(1) << 24), DP_EUNSUPPORTED);
    return DP_OK;
}

bool act_ok(dp_act act) { return act == DP_ACT_SILU || act == DP_ACT_GELU_TANH; }

}  // namespace
}  // namespace dpg

using namespace dpg;

namespace {

// few rows, and (bf16) up to kFfnRowsMax of them whose operands the tiles would have to pad
bool by_rows(const void *X, const void *Wg, const void *Wu, dp_dtype dt, i64 M, i64 K)
{
    if (dt == DP_F32 || M <= kFfnRowsBf16) return M <= kFfnRowsMax;
    return M <= kFfnRowsMax && !(K % 8 == 0 && ffn_tiles_ok(X, K) && ffn_tiles_ok(Wg, K) && ffn_tiles_ok(Wu, K));
}

}  // namespace

extern "C" size_t dp_gated_ffn_forward_workspace_bytes(int64_t M, int64_t d_in, int64_t d_ff, dp_dtype dt)
{
    if (!dtype_ok(dt) || check_sizes(M, d_in, d_ff) != DP_OK || M <= kFfnRowsMax) return 0;
    return dt == DP_BF16 ? ffn_bf16_forward_workspace(M, d_in, d_ff) : ffn_parts_forward_workspace(M, d_in, d_ff);
}

extern "C" dp_status dp_gated_ffn_forward(const void *X, const void *Wg, const void *Wu, dp_dtype dt, int64_t M,
                                          int64_t d_in, int64_t d_ff, dp_act act, void *H, void *G, void *U, void *ws,
                                          size_t ws_bytes, hipStream_t stream)
{
    DPG_REQUIRE(dtype_ok(dt), DP_EDTYPE);
    DPG_REQUIRE(act_ok(act), DP_EINVAL);
    const dp_status bad = check_sizes(M, d_in, d_ff);
    if (bad != DP_OK) return bad;
    if (M == 0) return DP_OK;
    DPG_REQUIRE(X != nullptr && Wg != nullptr && Wu != nullptr && H != nullptr, DP_EINVAL);
    DPG_REQUIRE((G == nullptr) == (U == nullptr), DP_EINVAL);
    const size_t need = dp_gated_ffn_forward_workspace_bytes(M, d_in, d_ff, dt);
    DPG_REQUIRE(need == 0 || (ws != nullptr && aligned(ws, 16) && ws_bytes >= need), DP_EINVAL);
    if (by_rows(X, Wg, Wu, dt, M, d_in)) {
        ffn_rows_forward(X, Wg, Wu, dt, M, d_in, d_ff, act, H, G, U, stream);
    } else if (dt == DP_F32) {
        ffn_parts_forward((const float *)X, (const float *)Wg, (const float *)Wu, M, d_in, d_ff, act, (float *)H, (float *)G,
                          (float *)U, ws, stream);
    } else {
        const uint16_t *x = (const uint16_t *)X, *wg = (const uint16_t *)Wg, *wu = (const uint16_t *)Wu;
        uint16_t *h = (uint16_t *)H, *g = (uint16_t *)G, *u = (uint16_t *)U;
        if (ffn_tiles_ok(X, d_in) && ffn_tiles_ok(Wg, d_in) && ffn_tiles_ok(Wu, d_in))
            ffn_bf16_forward(x, wg, wu, M, d_in, d_ff, act, h, g, u, ws, stream);
        else if (act == DP_ACT_SILU) forward_any<DP_ACT_SILU>(x, wg, wu, M, d_in, d_ff, h, g, u, stream);
        else forward_any<DP_ACT_GELU_TANH>(x, wg, wu, M, d_in, d_ff, h, g, u, stream);
    }
    return launch_status();
}

extern "C" size_t dp_gated_ffn_backward_workspace_bytes(int64_t M, int64_t d_in, int64_t d_ff, dp_dtype dt)
{
    if (!dtype_ok(dt) || check_sizes(M, d_in, d_ff) != DP_OK || M == 0) return 0;
    if (dt == DP_BF16) return ffn_bf16_dx_workspace(M, d_in, d_ff);
    return M <= kFfnRowsMax ? ffn_rows_dx_workspace(M, d_in, d_ff) : ffn_parts_dx_workspace(M, d_in, d_ff);
}

extern "C" dp_status dp_gated_ffn_backward(const void *dH, const void *G, const void *U, const void *Wg,
                                           const void *Wu, dp_dtype dt, int64_t M, int64_t d_in, int64_t d_ff,
                                           dp_act act, void *BG, void *BU, void *dX, void *ws, size_t ws_bytes,
                                           hipStream_t stream)
{
    DPG_REQUIRE(dtype_ok(dt), DP_EDTYPE);
    DPG_REQUIRE(act_ok(act), DP_EINVAL);
    const dp_status bad = check_sizes(M, d_in, d_ff);
    if (bad != DP_OK) return bad;
    if (M == 0) return DP_OK;
    DPG_REQUIRE(dH != nullptr && G != nullptr && U != nullptr && BG != nullptr && BU != nullptr && BG != BU, DP_EINVAL);
    DPG_REQUIRE(dX == nullptr || (Wg != nullptr && Wu != nullptr), DP_EINVAL);
    const size_t need = dX == nullptr ? 0 : dp_gated_ffn_backward_workspace_bytes(M, d_in, d_ff, dt);
    DPG_REQUIRE(need == 0 || (ws != nullptr && aligned(ws, 16) && ws_bytes >= need), DP_EINVAL);
    const i64 n = M * d_ff;
    if (dt == DP_F32) {
        if (act == DP_ACT_SILU) backprops<float, DP_ACT_SILU>(dH, G, U, n, BG, BU, stream);
        else backprops<float, DP_ACT_GELU_TANH>(dH, G, U, n, BG, BU, stream);
        if (dX == nullptr) return launch_status();
        if (M <= kFfnRowsMax) {
            ffn_rows_dx((const float *)BG, (const float *)BU, (const float *)Wg, (const float *)Wu, M, d_in, d_ff,
                        (float *)dX, ws, stream);
        } else {
            ffn_parts_dx((const float *)BG, (const float *)BU, (const float *)Wg, (const float *)Wu, M, d_in, d_ff,
                         (float *)dX, ws, stream);
        }
    } else {
        if (act == DP_ACT_SILU) backprops<uint16_t, DP_ACT_SILU>(dH, G, U, n, BG, BU, stream);
        else backprops<uint16_t, DP_ACT_GELU_TANH>(dH, G, U, n, BG, BU, stream);
        if (dX == nullptr) return launch_status();
        const uint16_t *bg = (const uint16_t *)BG, *bu = (const uint16_t *)BU;
        const uint16_t *wg = (const uint16_t *)Wg, *wu = (const uint16_t *)Wu;
        if (ffn_tiles_ok(BG, d_ff) && ffn_tiles_ok(BU, d_ff) && ffn_tiles_ok(Wg, d_in) && ffn_tiles_ok(Wu, d_in))
            ffn_bf16_dx(bg, bu, wg, wu, M, d_in, d_ff, (uint16_t *)dX, ws, stream);
        else
            dx_any(bg, bu, wg, wu, M, d_in, d_ff, (uint16_t *)dX, stream);
    }
    return launch_status();
}
