// The gated feed-forward block over few rows (ffn_rows.hip).
#pragma once

#include "common.hpp"

namespace dpg {

constexpr i64 kFfnRowsMax = 64;      // rows of X
constexpr i64 kFfnRowsBf16 = 16;     // above them the bf16 tiles are ahead (64 x 4096 -> 11008: 44 us, 81 here)

// H (and G, U unless NULL) from X [M][K], Wg, Wu [F][K], M <= kFfnRowsMax
void ffn_rows_forward(const void *X, const void *Wg, const void *Wu, dp_dtype dt, i64 M, i64 K, i64 F, dp_act act,
                      void *H, void *G, void *U, hipStream_t stream);

// dX [M][D] = BG Wg + BU Wu in fp32, M <= kFfnRowsMax; ws:
// ffn_rows_dx_workspace bytes, 16-byte aligned
size_t ffn_rows_dx_workspace(i64 M, i64 D, i64 F);
void ffn_rows_dx(const float *BG, const float *BU, const float *Wg, const float *Wu, i64 M, i64 D, i64 F, float *dX,
                 void *ws, hipStream_t stream);

}  // namespace dpg
