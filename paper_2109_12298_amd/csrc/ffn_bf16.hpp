// The bf16 tile kernels of the gated feed-forward block (ffn_bf16.hip).
#pragma once

#include "common.hpp"

namespace dpg {

// X, Wg and Wu as the tile kernels read them: rows of 16-byte pieces
inline bool ffn_rows_ok(const void *p, i64 cols) { return cols % 8 == 0 && aligned(p, 16); }

// H (and G, U unless NULL) from X [M][K], Wg, Wu [F][K] (ffn_rows_ok each)
void ffn_bf16_forward(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, dp_act act,
                      uint16_t *H, uint16_t *G, uint16_t *U, hipStream_t stream);

}  // namespace dpg
