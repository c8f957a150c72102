// Tiles of the gated feed-forward block for any size, type and alignment: 64 x
// 64, element loads, fp32 MFMA (products of bf16 values are exact in fp32).
// The work of the calls and values that the tile kernels of ffn_bf16.hip and
// ffn_parts.hip do not take.  THREADS threads stage, the first four waves multiply.
#pragma once

#include "gated_ffn.hpp"
#include "mfma_tile.hpp"

namespace dpg {
namespace ffn {

constexpr int kTM = 64, kTN = 64, kTK = 16;
constexpr int kLd = kTM + 1;              // LDS row: operands lie K-major, their loads come along K
constexpr int kAnyFloats = 3 * kTK * kLd; // LDS of a tile

// rows r0 .. r0+63 of P [rows][K], columns k0 .. k0+kTK-1, into L [kTK][kLd]; zeros outside
template <int THREADS, typename T>
__device__ __forceinline__ void stage_rows(const T *__restrict__ P, i64 rows, i64 K, i64 r0, i64 k0, float *L)
{
#pragma unroll
    for (int q = 0; q < kTM * kTK / THREADS; ++q) {
        const int e = threadIdx.x + THREADS * q;
        const int r = e / kTK, k = e % kTK;
        L[k * kLd + r] = r0 + r < rows && k0 + k < K ? load_elem<T>(P, (r0 + r) * K + k0 + k) : 0.0f;
    }
}

// rows k0 .. k0+kTK-1 of P [K][cols], columns c0 .. c0+63, into L [kTK][kLd]
template <int THREADS, typename T>
__device__ __forceinline__ void stage_cols(const T *__restrict__ P, i64 K, i64 cols, i64 k0, i64 c0, float *L)
{
#pragma unroll
    for (int q = 0; q < kTN * kTK / THREADS; ++q) {
        const int e = threadIdx.x + THREADS * q;
        const int k = e / kTN, c = e % kTN;
        L[k * kLd + c] = k0 + k < K && c0 + c < cols ? load_elem<T>(P, (k0 + k) * cols + c0 + c) : 0.0f;
    }
}

// H (and G, U) of positions m0 .. m0+63, features f0 .. f0+63
template <int THREADS, int ACT, typename T>
__device__ void any_forward_tile(const T *__restrict__ X, const T *__restrict__ Wg, const T *__restrict__ Wu, i64 M, i64 K,
                                 i64 F, i64 m0, i64 f0, T *__restrict__ H, T *__restrict__ G, T *__restrict__ U,
                                 float *lds)
{
    float *Xs = lds, *Gs = lds + kTK * kLd, *Us = lds + 2 * kTK * kLd;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave >> 1 & 1) * 32, wf = (wave & 1) * 32;
    const int li = lane & 31, lk = lane >> 5;
    f32x16 ag, au;
#pragma unroll
    for (int r = 0; r < 16; ++r) ag[r] = au[r] = 0.0f;
    for (i64 k0 = 0; k0 < K; k0 += kTK) {
        __syncthreads();
        stage_rows<THREADS>(X, M, K, m0, k0, Xs);
        stage_rows<THREADS>(Wg, F, K, f0, k0, Gs);
        stage_rows<THREADS>(Wu, F, K, f0, k0, Us);
        __syncthreads();
        if (wave >= 4) continue;
#pragma unroll
        for (int kk = 0; kk < kTK; kk += 2) {
            const float x = Xs[(kk + lk) * kLd + wm + li];
            ag = __builtin_amdgcn_mfma_f32_32x32x2f32(x, Gs[(kk + lk) * kLd + wf + li], ag, 0, 0, 0);
            au = __builtin_amdgcn_mfma_f32_32x32x2f32(x, Us[(kk + lk) * kLd + wf + li], au, 0, 0, 0);
        }
    }
    const i64 f = f0 + wf + li;
    if (wave >= 4 || f >= F) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const i64 m = m0 + wm + 8 * (r >> 2) + 4 * lk + (r & 3);
        if (m >= M) continue;
        store_elem(H + m * F + f, act<ACT>(ag[r]) * au[r]);
        if (G != nullptr) {
            store_elem(G + m * F + f, ag[r]);
            store_elem(U + m * F + f, au[r]);
        }
    }
}

// dX of positions m0 .. m0+63, columns d0 .. d0+63
template <int THREADS, typename T>
__device__ void any_dx_tile(const T *__restrict__ BG, const T *__restrict__ BU, const T *__restrict__ Wg,
                            const T *__restrict__ Wu, i64 M, i64 D, i64 F, i64 m0, i64 d0, T *__restrict__ dX, float *lds)
{
    float *Bs = lds, *Ws = lds + kTK * kLd;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave >> 1 & 1) * 32, wd = (wave & 1) * 32;
    const int li = lane & 31, lk = lane >> 5;
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    for (int half = 0; half < 2; ++half) {
        const T *P = half == 0 ? BG : BU, *W = half == 0 ? Wg : Wu;
        for (i64 k0 = 0; k0 < F; k0 += kTK) {
            __syncthreads();
            stage_rows<THREADS>(P, M, F, m0, k0, Bs);
            stage_cols<THREADS>(W, F, D, k0, d0, Ws);
            __syncthreads();
            if (wave >= 4) continue;
#pragma unroll
            for (int kk = 0; kk < kTK; kk += 2)
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(Bs[(kk + lk) * kLd + wm + li], Ws[(kk + lk) * kLd + wd + li],
                                                           acc, 0, 0, 0);
        }
    }
    const i64 d = d0 + wd + li;
    if (wave >= 4 || d >= D) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const i64 m = m0 + wm + 8 * (r >> 2) + 4 * lk + (r & 3);
        if (m < M) store_elem(dX + m * D + d, acc[r]);
    }
}

}  // namespace ffn
}  // namespace dpg
