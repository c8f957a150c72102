// Attention forward: the choice of shape, and the kernels for bf16.
#include "attention_forward_kernel.hpp"
#include "attention_order.hpp"

namespace dpg {
namespace attn {

dp_status forward_bf16(const Call &c, const ForwardOut &out, bool small, hipStream_t stream)
{
    return tiles_of<uint16_t>(c, out, small, stream);
}

namespace {

// Workgroups over which a sample's keys are split (1: none; 0: rows are blocks of 128).
int forward_splits(const dp_attention &a)
{
    const i64 M = a.Tq * (a.Hq / a.Hk), heads = a.N * a.Hk;
    if (M == 0 || heads == 0 || a.Tk == 0) return 1;
    if (M > 64 && heads * ceil_div(M, 128) >= 256) return 0;
    const i64 blocks = heads * ceil_div(M, 32);
    // workgroups for every CU, each at least a tile of keys for every wave; where there are many keys more of them, as samples may
    // differ in length
    i64 splits = ceil_div(256, blocks), more = ceil_div(1024, blocks);
    if (more > a.Tk / 512) more = a.Tk / 512;
    if (splits < more) splits = more;
    const i64 most = ceil_div(a.Tk, 4 * 32);
    if (splits > most) splits = most;
    return (int)(splits < 1 ? 1 : splits);
}

}  // namespace

size_t tiles_forward_workspace(const dp_attention &a)
{
    const i64 splits = forward_splits(a);
    if (splits == 0) return sizeof(int32_t) * (size_t)row_order_entries(a);
    return splits == 1 ? 0 : sizeof(float) * (size_t)(splits * a.N * a.Hq * a.Tq * (a.D + 2));
}

dp_status tiles_forward(const dp_attention &a, const Call &c, dp_dtype dt, void *O, float *lse, void *ws, hipStream_t stream)
{
    const int splits = forward_splits(a);
    ForwardOut out = {O, lse, (float *)ws, (i64)c.N * c.Hq * c.Tq, splits > 1 ? splits : 1, nullptr};
    if (splits == 0 && row_order_entries(a) > 0) {
        out.order = (const int32_t *)ws;
        order_blocks(c, (int32_t *)ws, nullptr, stream);
    }
    return dt == DP_F32 ? forward_f32(c, out, splits > 0, stream) : forward_bf16(c, out, splits > 0, stream);
}

}  // namespace attn
}  // namespace dpg
