// Attention backward: the choice of shapes, and the kernels for bf16.
#include "attention_backward_kernel.hpp"
#include "attention_order.hpp"

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

namespace {

struct Plan {
    bool small_q, small_k;
    i64 splits, info, part, row_order, key_order;        // and elements of each part of the workspace, all of 4 bytes
    explicit Plan(const dp_attention &a)
    {
        const i64 heads = a.N * a.Hk, G = a.Hq / a.Hk;
        small_q = small_blocks(heads, a.Tq * G);
        small_k = small_blocks(heads, a.Tk);
        splits = key_splits(heads, a.Tk, G, a.Tq);
        info = a.N * a.Hq * padded_queries(a.Tq);
        part = splits > 1 ? splits * heads * a.Tk * 2 * a.D : 0;
        row_order = small_q ? 0 : row_order_entries(a);
        key_order = small_k || a.Tq == 0 ? 0 : key_order_entries(a);
    }
};

}  // namespace

size_t tiles_backward_workspace(const dp_attention &a)
{
    if (a.N == 0 || a.Tq == 0) return 0;
    const Plan p(a);
    return 4 * (size_t)(2 * p.info + p.part + p.row_order + p.key_order);
}

dp_status tiles_backward(const dp_attention &a, const Call &c, dp_dtype dt, Grads g, void *ws, hipStream_t stream)
{
    const Plan p(a);
    g.pad = padded_queries(c.Tq);
    g.row_lse = (float *)ws;
    g.row_delta = g.row_lse + p.info;
    g.part = g.row_delta + p.info;
    int32_t *rows = (int32_t *)(g.part + p.part), *keys = rows + p.row_order;
    g.row_order = rows = p.row_order > 0 ? rows : nullptr;
    g.key_order = keys = p.key_order > 0 ? keys : nullptr;
    g.small_q = p.small_q;
    g.small_k = p.small_k;
    g.splits = (int)p.splits;
    if (c.Tq > 0) order_blocks(c, rows, keys, stream);
    return dt == DP_F32 ? backward_f32(c, g, stream) : backward_bf16(c, g, stream);
}

}  // namespace attn
}  // namespace dpg
