// Attention's entry points: argument checks and the choice of kernels.
#include "attention.hpp"
#include "attention_backward.hpp"
#include "attention_forward.hpp"

#include <math.h>

using namespace dpg;
using namespace dpg::attn;

namespace {

constexpr i64 kMaxT = i64(1) << 24, kMaxRows = i64(1) << 31, kMaxLd = i64(1) << 22,
              kMaxBlocks = i64(1) << 24;

dp_status check(const dp_attention *a)
{
    DPG_REQUIRE(a != nullptr, DP_EINVAL);
    DPG_REQUIRE(a->dt == DP_F32 || a->dt == DP_BF16, DP_EDTYPE);
    DPG_REQUIRE((a->flags & ~(uint32_t)(DP_ATTENTION_CAUSAL | DP_ATTENTION_LAST)) == 0, DP_EINVAL);
    DPG_REQUIRE(a->N >= 0 && a->Tq >= 0 && a->Tk >= 0 && a->Hk >= 1 && a->Hq >= 1 && a->Hq % a->Hk == 0 && a->D >= 1,
                DP_EINVAL);
    // within these bounds scale / softcap and the scales in units of ln 2 are finite
    DPG_REQUIRE(fabsf(a->scale) <= 0x1p60f && (a->softcap == 0.0f || (a->softcap >= 0x1p-60f && a->softcap <= 0x1p60f)), DP_EINVAL);
    DPG_REQUIRE(a->prefix == nullptr || (a->flags & DP_ATTENTION_CAUSAL) != 0, DP_EINVAL);
    DPG_REQUIRE(aligned(a->slopes, 4) && aligned(a->lens, 4) && aligned(a->prefix, 4) && aligned(a->docs, 4), DP_EINVAL);
    DPG_REQUIRE(a->D <= kMaxD && a->Tq < kMaxT && a->Tk < kMaxT && a->N < kMaxRows && a->Hq < kMaxLd, DP_EUNSUPPORTED);
    DPG_REQUIRE(a->N * a->Hq < kMaxRows, DP_EUNSUPPORTED);
    // a dimension of a grid holds fewer than 2^32 threads, and 32 queries or keys of a head are a workgroup at the least
    DPG_REQUIRE(a->N * a->Hq * ceil_div(a->Tq, 32) < kMaxBlocks && a->N * a->Hk * ceil_div(a->Tk, 32) < kMaxBlocks,
                DP_EUNSUPPORTED);
    DPG_REQUIRE(a->ldq >= a->Hq * a->D && a->ldo >= a->Hq * a->D && a->ldk >= a->Hk * a->D && a->ldv >= a->Hk * a->D, DP_EINVAL);
    DPG_REQUIRE(a->ldq < kMaxLd && a->ldo < kMaxLd && a->ldk < kMaxLd && a->ldv < kMaxLd, DP_EUNSUPPORTED);
    return DP_OK;
}

Call call_of(const dp_attention &a, const void *Q, const void *K, const void *V)
{
    return {Q,     K,     V,     (int)a.N, (int)a.Tq, (int)a.Tk, (int)a.Hq,  (int)a.Hk, (int)a.D, (int)(a.Hq / a.Hk),
            a.ldq, a.ldk, a.ldv, a.ldo,    a.scale,   a.softcap, a.slopes,   a.lens,    a.prefix, a.docs,
            (a.flags & DP_ATTENTION_CAUSAL) != 0, (a.flags & DP_ATTENTION_LAST) != 0};
}

}  // namespace

extern "C" size_t dp_attention_forward_workspace_bytes(const dp_attention *a)
{
    if (check(a) != DP_OK || a->D > kTileD) return 0;
    return tiles_forward_workspace(*a);
}

extern "C" dp_status dp_attention_forward(const dp_attention *a, const void *Q, const void *K, const void *V, void *O,
                                          float *lse, void *ws, size_t ws_bytes, hipStream_t stream)
{
    const dp_status s = check(a);
    if (s != DP_OK) return s;
    if (a->N == 0 || a->Tq == 0) return DP_OK;
    const size_t e = dtype_bytes((dp_dtype)a->dt);
    DPG_REQUIRE(Q != nullptr && O != nullptr && (a->Tk == 0 || (K != nullptr && V != nullptr)), DP_EINVAL);
    DPG_REQUIRE(aligned(Q, e) && aligned(K, e) && aligned(V, e) && aligned(O, e) && aligned(lse, 4), DP_EINVAL);
    const size_t need = dp_attention_forward_workspace_bytes(a);
    DPG_REQUIRE(need == 0 || (ws != nullptr && aligned(ws, 16) && ws_bytes >= need), DP_EINVAL);
    const Call c = call_of(*a, Q, K, V);
    if (a->D > kTileD) return rows_forward(c, (dp_dtype)a->dt, O, lse, stream);
    return tiles_forward(*a, c, (dp_dtype)a->dt, O, lse, ws, stream);
}

extern "C" size_t dp_attention_backward_workspace_bytes(const dp_attention *a)
{
    if (check(a) != DP_OK) return 0;
    return a->D > kTileD ? sizeof(float) * (size_t)(a->N * a->Hq * a->Tq) : tiles_backward_workspace(*a);
}

extern "C" dp_status dp_attention_backward(const dp_attention *a, const void *Q, const void *K, const void *V,
                                           const void *O, const float *lse, const void *dO, void *dQ, void *dK, void *dV,
                                           void *ws, size_t ws_bytes, hipStream_t stream)
{
    const dp_status s = check(a);
    if (s != DP_OK) return s;
    if (a->N == 0 || (a->Tq == 0 && a->Tk == 0)) return DP_OK;
    const size_t e = dtype_bytes((dp_dtype)a->dt);
    DPG_REQUIRE(a->Tq == 0 || (Q != nullptr && O != nullptr && lse != nullptr && dO != nullptr && dQ != nullptr), DP_EINVAL);
    DPG_REQUIRE(a->Tk == 0 || (K != nullptr && V != nullptr && dK != nullptr && dV != nullptr), DP_EINVAL);
    DPG_REQUIRE(a->Tk == 0 || dK != dV, DP_EINVAL);
    DPG_REQUIRE(aligned(Q, e) && aligned(K, e) && aligned(V, e) && aligned(O, e) && aligned(lse, 4) && aligned(dO, e) &&
                    aligned(dQ, e) && aligned(dK, e) && aligned(dV, e),
                DP_EINVAL);
    const size_t need = dp_attention_backward_workspace_bytes(a);
    DPG_REQUIRE(need == 0 || (ws != nullptr && aligned(ws, 16) && ws_bytes >= need), DP_EINVAL);
    const Call c = call_of(*a, Q, K, V);
    if (a->D > kTileD) return rows_backward(c, (dp_dtype)a->dt, O, lse, dO, dQ, dK, dV, ws, stream);
    return tiles_backward(*a, c, (dp_dtype)a->dt, {O, dO, lse, dQ, dK, dV}, ws, stream);
}
