// Attention forward for fp32.
#include "attention_forward_kernel.hpp"

namespace dpg {
namespace attn {

dp_status forward_f32(const Call &c, const ForwardOut &out, bool small, hipStream_t stream)
{
    return tiles_of<float>(c, out, small, stream);
}

}  // namespace attn
}  // namespace dpg
