// Attention backward: the choice of shapes, and the kernels for bf16.
#include "attention_backward_kernel.hpp"

namespace dpg {
namespace attn {

namespace {

int padded_queries(i64 Tq) { return (int)((Tq + 63) / 64 * 64); }

}  // namespace

dp_status backward_bf16(const Call &c, const Grads &g, hipStream_t stream) { return tiles_of<uint16_t>(c, g, stream); }

size_t tiles_backward_workspace(const dp_attention &a)
{
    if (a.N == 0 || a.Tq == 0) return 0;
    return 2 * sizeof(float) * (size_t)(a.N * a.Hq * padded_queries(a.Tq));
}

dp_status tiles_backward(const Call &c, dp_dtype dt, Grads g, void *ws, hipStream_t stream)
{
    g.pad = padded_queries(c.Tq);
    g.row_lse = (float *)ws;
    g.row_delta = g.row_lse + (i64)c.N * c.Hq * g.pad;
    const i64 heads = (i64)c.N * c.Hk;
    g.small_q = heads * ceil_div((i64)c.Tq * c.G, 128) < 256;
    g.small_k = heads * ceil_div(c.Tk, 128) < 256;
    return dt == DP_F32 ? backward_f32(c, g, stream) : backward_bf16(c, g, stream);
}

}  // namespace attn
}  // namespace dpg
