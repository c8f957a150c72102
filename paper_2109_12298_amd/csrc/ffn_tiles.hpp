// What the tile kernels of the gated feed-forward block share (ffn_bf16.hip,
// ffn_parts.hip): staging loads, tile order, output stores.
#pragma once

#include "bf16_stage.hpp"
#include "gated_ffn.hpp"

namespace dpg {
namespace {

using namespace bf16s;
using namespace ffn;

// lane l's 16 bytes at base + off go to LDS byte lds + 16 l (see dma16); STREAM:
// past the caches
template <bool STREAM = false>
__device__ __forceinline__ void dma16_off(const void *base, uint32_t off, uint32_t lds)
{
    if constexpr (STREAM)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base),
                     "s"(__builtin_amdgcn_readfirstlane(lds))
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base),
                     "s"(__builtin_amdgcn_readfirstlane(lds))
                     : "memory", "m0");
}

// Tile order: workgroups go round robin over the XCDs; each XCD takes a run of
// consecutive tiles, 8 tiles of positions by as many tiles of features as the
// run holds, so that its L2 serves the operand rows that they share.
__device__ __forceinline__ void tile_of(int b, int nb, int tiles_m, int tiles_n, int &tm, int &tn)
{
    constexpr int GM = 8;
    const int t = (int)xcd_swizzle32((uint32_t)b, (uint32_t)nb);
    const int group = t / (GM * tiles_n), m0 = group * GM;
    const int gm = tiles_m - m0 < GM ? tiles_m - m0 : GM;
    const int in = t - group * GM * tiles_n;
    tm = m0 + in % gm;
    tn = in / gm;
}

// 32 rows by COLS values of one output tile, from LDS rows of LDT bytes
template <typename T, int COLS, int LDT>
__device__ __forceinline__ void store_rows(const char *L, T *__restrict__ O, i64 rows, i64 cols, i64 r0, i64 c0, bool vec,
                                           int lane)
{
    // LDS reads ahead of the stores, whose bounds are branches
    if (vec) {                            // 16-byte pieces
        constexpr int N = 16 / sizeof(T), LPR = COLS / N, RPS = 64 / LPR;    // values per piece, lanes per row, rows per store
        uint4 v[32 / RPS];
#pragma unroll
        for (int s = 0; s < 32 / RPS; ++s)
            v[s] = *reinterpret_cast<const uint4 *>(L + (s * RPS + lane / LPR) * LDT + 16 * (lane % LPR));
#pragma unroll
        for (int s = 0; s < 32 / RPS; ++s) {
            const i64 r = r0 + s * RPS + lane / LPR, f = c0 + N * (lane % LPR);
            if (r < rows && f < cols) *reinterpret_cast<uint4 *>(O + r * cols + f) = v[s];
        }
    } else {                              // rows of any alignment: 64 consecutive values per store
        constexpr int STORES = 32 * COLS / 64, AHEAD = 16;
        static_assert(STORES % AHEAD == 0, "whole batches");
        for (int s0 = 0; s0 < STORES; s0 += AHEAD) {
            T v[AHEAD];
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const int e = 64 * (s0 + s) + lane;
                v[s] = *reinterpret_cast<const T *>(L + e / COLS * LDT + (int)sizeof(T) * (e % COLS));
            }
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const int e = 64 * (s0 + s) + lane;
                const i64 r = r0 + e / COLS, f = c0 + e % COLS;
                if (r < rows && f < cols) O[r * cols + f] = v[s];
            }
        }
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    return (uint32_t)bf16_bits(a) | ((uint32_t)bf16_bits(b) << 16);
}

// four consecutive values of a row to LDS
__device__ __forceinline__ void put4(uint16_t *p, float a, float b, float c, float d)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(a, b), pack2(c, d));
}
__device__ __forceinline__ void put4(float *p, float a, float b, float c, float d)
{
    *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d);
}

inline i64 padded(i64 cols) { return (cols + 7) / 8 * 8; }

}  // namespace
}  // namespace dpg
