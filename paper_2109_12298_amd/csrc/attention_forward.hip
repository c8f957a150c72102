// Attention forward: the choice of shape, and the kernels for bf16.
#include "attention_forward_kernel.hpp"

namespace dpg {
namespace attn {

dp_status forward_bf16(const Call &c, const ForwardOut &out, bool small, hipStream_t stream)
{
    return tiles_of<uint16_t>(c, out, small, stream);
}

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

size_t tiles_forward_workspace(const dp_attention &a)
{
    const i64 splits = forward_splits(a);
    if (splits <= 1) return 0;
    return sizeof(float) * (size_t)(splits * a.N * a.Hq * a.Tq * (a.D + 2));
}

dp_status tiles_forward(const Call &c, dp_dtype dt, int splits, void *O, float *lse, void *ws, hipStream_t stream)
{
    const ForwardOut out = {O, lse, (float *)ws, (i64)c.N * c.Hq * c.Tq, splits > 1 ? splits : 1};
    return dt == DP_F32 ? forward_f32(c, out, splits > 0, stream) : forward_bf16(c, out, splits > 0, stream);
}

}  // namespace attn
}  // namespace dpg
