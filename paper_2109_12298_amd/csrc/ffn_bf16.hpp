// The tile kernels of the gated feed-forward block (ffn_bf16.hip, ffn_parts.hip).
#pragma once

#include "common.hpp"

namespace dpg {

// Operands as the tile kernels take them: rows of any length from a 16-byte
// boundary (rows that are no multiple of 16 bytes are padded into the
// workspace first), row offsets of a tile in 32 bits.
constexpr i64 kFfnTilesMax = i64(1) << 21;
inline bool ffn_tiles_ok(const void *p, i64 cols) { return aligned(p, 16) && cols < kFfnTilesMax; }

// H (and G, U unless NULL) from X [M][K], Wg, Wu [F][K] (ffn_tiles_ok each);
// ws: ffn_bf16_forward_workspace bytes, 16-byte aligned
size_t ffn_bf16_forward_workspace(i64 M, i64 K, i64 F);
void ffn_bf16_forward(const uint16_t *X, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 K, i64 F, dp_act act,
                      uint16_t *H, uint16_t *G, uint16_t *U, void *ws, hipStream_t stream);

// dX [M][D] = BG Wg + BU Wu from BG, BU [M][F] and Wg, Wu [F][D] (ffn_tiles_ok
// each); ws: ffn_bf16_dx_workspace bytes, 16-byte aligned
size_t ffn_bf16_dx_workspace(i64 M, i64 D, i64 F);
void ffn_bf16_dx(const uint16_t *BG, const uint16_t *BU, const uint16_t *Wg, const uint16_t *Wu, i64 M, i64 D, i64 F,
                 uint16_t *dX, void *ws, hipStream_t stream);

// The same for fp32 values, each as three bf16 parts and every product as six
// bf16 products (what is left out is 2^-24 of a product), M > kFfnRowsMax.
// Rows of any length and alignment (the splitting kernel lays them out anew).
// Tiles whose sums come out non-finite (infinities, NaN, magnitudes from about
// 2^104 on, sums from 2^80 on) are formed again on the fp32 units (ffn_any.hpp),
// inside the same launches.
size_t ffn_parts_forward_workspace(i64 M, i64 K, i64 F);
void ffn_parts_forward(const float *X, const float *Wg, const float *Wu, i64 M, i64 K, i64 F, dp_act act, float *H,
                       float *G, float *U, void *ws, hipStream_t stream);
size_t ffn_parts_dx_workspace(i64 M, i64 D, i64 F);
void ffn_parts_dx(const float *BG, const float *BU, const float *Wg, const float *Wu, i64 M, i64 D, i64 F, float *dX,
                  void *ws, hipStream_t stream);

}  // namespace dpg
