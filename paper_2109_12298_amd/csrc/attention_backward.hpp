// Attention backward on tiles: see attention_backward_kernel.hpp.
#pragma once

#include "attention.hpp"

namespace dpg {
namespace attn {

struct Grads {
    const void *O, *dO;
    const float *lse;
    void *dQ, *dK, *dV;
    float *row_lse, *row_delta;      // [N][Hq][pad]: lse in units of ln 2 (+inf: the query sees nothing), dO.O
    int pad;                         // queries, rounded up to 64
    float *part;                     // [splits][N][Hk][Tk][2][D]: sums for dK and dV
    const int32_t *row_order, *key_order;      // when blocks of rows and of keys run, or NULL (attention_order.hip)
    bool small_q, small_k;           // 32 rows (keys) a workgroup instead of 128
    int splits;                      // workgroups over which a block of keys' queries are split (small_k)
};

size_t tiles_backward_workspace(const dp_attention &a);
dp_status tiles_backward(const dp_attention &a, const Call &c, dp_dtype dt, Grads g, void *ws, hipStream_t stream);

dp_status backward_bf16(const Call &c, const Grads &g, hipStream_t stream);
dp_status backward_f32(const Call &c, const Grads &g, hipStream_t stream);

}  // namespace attn
}  // namespace dpg
