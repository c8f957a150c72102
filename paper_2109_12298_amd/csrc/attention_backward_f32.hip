// Attention backward for fp32.
#include "attention_backward_kernel.hpp"

namespace dpg {
namespace attn {

dp_status backward_f32(const Call &c, const Grads &g, hipStream_t stream) { return tiles_of<float>(c, g, stream); }

}  // namespace attn
}  // namespace dpg
