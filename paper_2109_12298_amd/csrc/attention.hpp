// Shared by the attention kernels: the call as the kernels see it, positions,
// masks and scores.
#pragma once

#include "common.hpp"

namespace dpg {
namespace attn {

constexpr int kMaxD = 256, kTileD = 128;      // values of a head, at the most: at all, and in the tiles
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Call {
    const void *Q, *K, *V;
    int N, Tq, Tk, Hq, Hk, D, G;            // G = Hq / Hk query heads per key head
    i64 ldq, ldk, ldv, ldo;
    float scale, cap;
    const float *slopes;
    const int32_t *lens, *prefix, *docs;
    int causal, last;
};

// One sample's keys, positions and mask.
struct Sample {
    int L, first, prefix;                   // keys; position of query 0; keys that all its queries see
    const int32_t *docs;
    bool causal;

    __device__ __forceinline__ Sample(const Call &c, int n)
    {
        L = c.lens != nullptr ? c.lens[n] : c.Tk;
        L = L < 0 ? 0 : L > c.Tk ? c.Tk : L;
        first = c.last ? L - c.Tq : 0;
        prefix = c.prefix != nullptr ? c.prefix[n] : 0;
        docs = c.docs != nullptr ? c.docs + (i64)n * c.Tk : nullptr;
        causal = c.causal != 0;
    }
    // keys from here on are seen by no query at position <= p
    __device__ __forceinline__ int end_for(int p) const
    {
        if (p < 0) return 0;
        if (!causal) return L;
        const int e = p + 1 > prefix ? p + 1 : prefix;
        return e < L ? e : L;
    }
    __device__ __forceinline__ bool sees(int p, int j) const
    {
        bool v = p >= 0 && p < L && j < L && (!causal || j <= p || j < prefix);
        if (v && docs != nullptr) v = docs[j] == docs[p] && docs[p] >= 0;
        return v;
    }
};

// The score of q.k = x in units of ln 2 (so that its softmax takes exp2), and
// the derivative of the capped score by the uncapped one.
__device__ __forceinline__ float score2(const Call &c, float x, float slope, int far, float &slope_of_cap)
{
    float s = c.scale * x;
    slope_of_cap = 1.0f;
    if (c.cap > 0.0f) {
        // (1 - tanh^2 as a product: the difference would lose its digits where the cap is far exceeded)
        const float y = s / c.cap, e = expf(-2.0f * fabsf(y)), r = 1.0f / (1.0f + e);
        s = c.cap * tanhf(y);
        slope_of_cap = 4.0f * e * r * r;
    }
    s -= slope * (float)far;
    return s * kLog2e;
}

__device__ __forceinline__ uint16_t bf16_bits(float x)
{
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ void store_elem(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(uint16_t *p, float v) { *p = bf16_bits(v); }

__device__ __forceinline__ float wave_max(float v)
{
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, kWave));
    return v;
}

// host side: the kernels of attention_rows.hip (the backward ones' workspace: a float for each of N * Hq * Tq rows)
dp_status rows_forward(const Call &c, dp_dtype dt, void *O, float *lse, hipStream_t stream);
dp_status rows_backward(const Call &c, dp_dtype dt, const void *O, const float *lse, const void *dO, void *dQ, void *dK,
                        void *dV, void *ws, hipStream_t stream);

}  // namespace attn
}  // namespace dpg
