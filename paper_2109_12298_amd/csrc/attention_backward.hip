// Attention backward: the choice of shapes, and the kernels for bf16.
#include "attention_backward_kernel.hpp"

namespace dpg {
namespace attn {

namespace {

int padded_queries(i64 Tq) { return (int)((Tq + 63) / 64 * 64); }

bool small_blocks(i64 heads, i64 rows) { return heads * ceil_div(rows, 128) < 256; }

// Workgroups for every CU from the blocks of 32 keys, each with a tile of queries for every wave.
i64 key_splits(i64 heads, i64 Tk, i64 G, i64 Tq)
{
    if (Tk == 0 || Tq == 0 || !small_blocks(heads, Tk)) return 1;
    const i64 splits = ceil_div(256, heads * ceil_div(Tk, 32)), most = G * ceil_div(Tq, 32) / 4;
    return splits < most ? splits : most < 1 ? 1 : most;
}

}  // namespace

dp_status backward_bf16(const Call &c, const Grads &g, hipStream_t stream) { return tiles_of<uint16_t>(c, g, stream); }

size_t tiles_backward_workspace(const dp_attention &a)
{
    if (a.N == 0 || a.Tq == 0) return 0;
    const i64 splits = key_splits(a.N * a.Hk, a.Tk, a.Hq / a.Hk, a.Tq);
    return sizeof(float) * (size_t)(2 * a.N * a.Hq * padded_queries(a.Tq) + (splits > 1 ? splits * a.N * a.Hk * a.Tk * 2 * a.D : 0));
}

dp_status tiles_backward(const Call &c, dp_dtype dt, Grads g, void *ws, hipStream_t stream)
{
    const i64 heads = (i64)c.N * c.Hk;
    g.pad = padded_queries(c.Tq);
    g.row_lse = (float *)ws;
    g.row_delta = g.row_lse + (i64)c.N * c.Hq * g.pad;
    g.part = g.row_delta + (i64)c.N * c.Hq * g.pad;
    g.small_q = small_blocks(heads, (i64)c.Tq * c.G);
    g.small_k = small_blocks(heads, c.Tk);
    g.splits = (int)key_splits(heads, c.Tk, c.G, c.Tq);
    return dt == DP_F32 ? backward_f32(c, g, stream) : backward_bf16(c, g, stream);
}

}  // namespace attn
}  // namespace dpg
