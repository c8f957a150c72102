// Attention one row at a time, a wave to a row: right for every size, mask and
// value, as products are formed for visible pairs only.  Lanes take 64 keys (or
// queries) at a time for the scores, then a head's values for the sums.
#pragma once

#include "attention.hpp"

namespace dpg {
namespace attn {

constexpr int kPerLane = kMaxD / kWave;     // a head's values per lane

template <typename T>
__device__ __forceinline__ float dot(const T *a, const T *b, int D)
{
    float s = 0.0f;
    for (int d = 0; d < D; ++d) s += load_elem<T>(a, d) * load_elem<T>(b, d);
    return s;
}

// acc[k] += w_l * x_l[lane + 64 k] for the lanes l with take_l, in lane order
template <typename T>
__device__ __forceinline__ void add_rows(float (&acc)[kPerLane], bool take, float w, const T *base, i64 ld, int first, int step,
                                         int D)
{
    const int lane = threadIdx.x & (kWave - 1);
    unsigned long long left = __ballot(take);
    while (left != 0) {
        const int l = __ffsll(left) - 1;
        left &= left - 1;
        const float f = __shfl(w, l, kWave);
        const T *x = base + (i64)(first + l * step) * ld;
#pragma unroll
        for (int k = 0; k < kPerLane; ++k)
            if (lane + kWave * k < D) acc[k] += f * load_elem<T>(x, lane + kWave * k);
    }
}

// o of query i, head h of sample n; lse or NULL
template <typename T>
__device__ void forward_row(const Call &c, int n, int h, int i, T *O, float *lse)
{
    const int lane = threadIdx.x & (kWave - 1), kv = h / c.G;
    const Sample s(c, n);
    const int p = s.first + i, end = p < s.L ? s.end_for(p) : 0;
    const T *q = (const T *)c.Q + ((i64)n * c.Tq + i) * c.ldq + (i64)h * c.D;
    const T *K = (const T *)c.K + (i64)n * c.Tk * c.ldk + (i64)kv * c.D;
    const T *V = (const T *)c.V + (i64)n * c.Tk * c.ldv + (i64)kv * c.D;
    const float slope = c.slopes != nullptr ? c.slopes[h] : 0.0f;
    float acc[kPerLane] = {}, top = -INFINITY, sum = 0.0f;
    for (int j0 = 0; j0 < end; j0 += kWave) {
        const int j = j0 + lane;
        const bool see = j < end && s.sees(p, j);
        float x = -INFINITY, unused;
        if (see) x = score2(c, dot<T>(q, K + (i64)j * c.ldk, c.D), slope, p < j ? j - p : p - j, unused);
        const float t = fmaxf(top, wave_max(x));
        const float base = t == -INFINITY ? 0.0f : t;
        const float w = see ? exp2f(x - base) : 0.0f, f = exp2f(top - base);
        sum = sum * f + wave_sum(w);
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) acc[k] *= f;
        add_rows<T>(acc, see, w, V, c.ldv, j0, 1, c.D);
        top = t;
    }
    T *o = O + ((i64)n * c.Tq + i) * c.ldo + (i64)h * c.D;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k)
        if (lane + kWave * k < c.D) store_elem(o + lane + kWave * k, sum == 0.0f ? 0.0f : acc[k] / sum);
    if (lse != nullptr && lane == 0)
        lse[((i64)n * c.Hq + h) * c.Tq + i] = sum == 0.0f ? -INFINITY : top * kLn2 + logf(sum);
}

// p, e = p (dO.V - delta) and g of a visible pair of query i (head h) and key j; delta = dO.O of the query
template <typename T>
__device__ __forceinline__ void pair_grads(const Call &c, const T *q, const T *k, const T *v, const T *dO, float slope, int far,
                                           float lse, float delta, float &p, float &e, float &g)
{
    float bend;
    const float x = score2(c, dot<T>(q, k, c.D), slope, far, bend);
    p = lse == -INFINITY ? 0.0f : exp2f(x - lse * kLog2e);
    e = p * (dot<T>(dO, v, c.D) - delta);
    g = e * bend * c.scale;
}

// Two passes over the keys: O is rounded, and dO.O with it, so the first one adds up what p and dO.V say it lacks.  row_delta: where
// the sum goes, which backward_key_row takes, or NULL
template <typename T>
__device__ void backward_query_row(const Call &c, int n, int h, int i, const T *O, const float *lse, const T *dO, T *dQ,
                                   float *row_delta)
{
    const int lane = threadIdx.x & (kWave - 1), kv = h / c.G;
    const Sample s(c, n);
    const int p = s.first + i, end = p < s.L ? s.end_for(p) : 0;
    const i64 at = ((i64)n * c.Tq + i) * c.ldq + (i64)h * c.D, ato = ((i64)n * c.Tq + i) * c.ldo + (i64)h * c.D;
    const T *q = (const T *)c.Q + at;
    const T *K = (const T *)c.K + (i64)n * c.Tk * c.ldk + (i64)kv * c.D;
    const T *V = (const T *)c.V + (i64)n * c.Tk * c.ldv + (i64)kv * c.D;
    const float slope = c.slopes != nullptr ? c.slopes[h] : 0.0f;
    const float l = lse[((i64)n * c.Hq + h) * c.Tq + i];
    float delta = end > 0 && l != -INFINITY ? dot<T>(dO + ato, O + ato, c.D) : 0.0f, excess = 0.0f;
    float acc[kPerLane] = {};
    const auto pair = [&](int j, bool see, float &pr, float &e, float &g) {
        pr = e = g = 0.0f;
        if (see)
            pair_grads<T>(c, q, K + (i64)j * c.ldk, V + (i64)j * c.ldv, dO + ato, slope, p < j ? j - p : p - j, l, delta, pr, e, g);
    };
    float pr, e, g;
    for (int j = lane; j < end; j += kWave) {
        pair(j, s.sees(p, j), pr, e, g);
        excess += e;
    }
    delta += wave_sum(excess);
    if (row_delta != nullptr && lane == 0) *row_delta = delta;
    for (int j0 = 0; j0 < end; j0 += kWave) {
        const int j = j0 + lane;
        const bool see = j < end && s.sees(p, j);
        pair(j, see, pr, e, g);
        add_rows<T>(acc, see, g, K, c.ldk, j0, 1, c.D);
    }
#pragma unroll
    for (int k = 0; k < kPerLane; ++k)
        if (lane + kWave * k < c.D) store_elem(dQ + at + lane + kWave * k, acc[k]);
}

// dK, dV: either may be NULL; row_delta: [N][Hq][pad]
template <typename T>
__device__ void backward_key_row(const Call &c, int n, int kv, int j, const float *lse, const float *row_delta, int pad, const T *dO,
                                 T *dK, T *dV)
{
    const int lane = threadIdx.x & (kWave - 1);
    const Sample s(c, n);
    const T *k = (const T *)c.K + ((i64)n * c.Tk + j) * c.ldk + (i64)kv * c.D;
    const T *v = (const T *)c.V + ((i64)n * c.Tk + j) * c.ldv + (i64)kv * c.D;
    float ak[kPerLane] = {}, av[kPerLane] = {};
    if (j < s.L)
        for (int g = 0; g < c.G; ++g) {
            const int h = kv * c.G + g;
            const float slope = c.slopes != nullptr ? c.slopes[h] : 0.0f;
            const T *Q = (const T *)c.Q + (i64)n * c.Tq * c.ldq + (i64)h * c.D;
            const T *dOn = dO + (i64)n * c.Tq * c.ldo + (i64)h * c.D;
            for (int i0 = 0; i0 < c.Tq; i0 += kWave) {
                const int i = i0 + lane, p = s.first + i;
                const bool see = i < c.Tq && s.sees(p, j);
                float pr = 0.0f, e, gr = 0.0f;
                if (see)
                    pair_grads<T>(c, Q + (i64)i * c.ldq, k, v, dOn + (i64)i * c.ldo, slope, p < j ? j - p : p - j,
                                  lse[((i64)n * c.Hq + h) * c.Tq + i], row_delta[((i64)n * c.Hq + h) * pad + i], pr, e, gr);
                add_rows<T>(ak, see, gr, Q, c.ldq, i0, 1, c.D);
                add_rows<T>(av, see, pr, dOn, c.ldo, i0, 1, c.D);
            }
        }
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
        if (lane + kWave * e < c.D) {
            if (dK != nullptr) store_elem(dK + ((i64)n * c.Tk + j) * c.ldk + (i64)kv * c.D + lane + kWave * e, ak[e]);
            if (dV != nullptr) store_elem(dV + ((i64)n * c.Tk + j) * c.ldv + (i64)kv * c.D + lane + kWave * e, av[e]);
        }
}

}  // namespace attn
}  // namespace dpg
