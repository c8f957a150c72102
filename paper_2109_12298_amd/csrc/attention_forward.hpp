// Attention forward on tiles: see attention_forward_kernel.hpp.
#pragma once

#include "attention.hpp"

namespace dpg {
namespace attn {

struct ForwardOut {
    void *O;
    float *lse;
    float *part;             // [splits][rows][D], and behind it [splits][rows][2]: maximum and sum
    i64 rows;                // N * Hk * M
    int splits;
    const int32_t *order;    // [N * blocks of rows]: when they run, or NULL (attention_order.hip)
};

size_t tiles_forward_workspace(const dp_attention &a);
dp_status tiles_forward(const dp_attention &a, const Call &c, dp_dtype dt, void *O, float *lse, void *ws, hipStream_t stream);

dp_status forward_bf16(const Call &c, const ForwardOut &out, bool small, hipStream_t stream);
dp_status forward_f32(const Call &c, const ForwardOut &out, bool small, hipStream_t stream);

}  // namespace attn
}  // namespace dpg
