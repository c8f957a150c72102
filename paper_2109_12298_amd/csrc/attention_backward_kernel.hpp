// Attention backward: with s the scores, p = exp(s - lse) and delta = dO.O,
//   dV_j = sum_i p_ij dO_i,  e_ij = p_ij (dO_i.V_j - delta_i) (1 - tanh^2),
//   dQ_i = scale sum_j e_ij K_j,  dK_j = scale sum_i e_ij Q_i.
//
// Two launches: dQ (with lse and delta of every query, which the other reads), by
// blocks of rows over tiles of keys, as the forward pass; dK and dV, by blocks of
// keys over tiles of queries.  Scores and dO.V are formed in both (seven products
// where five would do), so that every sum belongs to one workgroup: no atomics, no
// partial sums in memory, the same bits every run, and a key head's sum over its query
// heads is one more loop.
//
// dQ forms scores as keys x rows and dK, dV as rows x keys, so that p and e are
// in either the second operand of the product that sums over them, in the
// registers they were formed in (attention_tile.hpp).  Blocks of 128 rows or
// keys share tiles, two stages deep, where there are blocks enough to fill the
// card; else 32 are one workgroup whose waves take different tiles and whose
// sums are added in wave order; few blocks of keys have their queries split over
// workgroups as well, and the splits' sums are added by a launch of their own (3
// samples of 500, 6 and 2 heads of 48, fp32: 96 blocks 70 us, split 31 + 5).
//
// With bf16 values O is rounded, and delta with it.  What it lacks, x_i = sum_j p_ij
// (dO_i.V_j - delta_i), is known once dQ's launch has been over all keys: dK's takes
// the whole delta, and dQ less scale x_i sum_j p_ij (1 - tanh^2) K_j, a second sum
// beside its own (p rounded to bf16 there, as x is some 2^-9 of dO.O).  A part that
// all keys share drops out of dQ, as e adds up to 0, but not while delta lacks x:
// dQ was then off by up to several times itself.  The second sum is a quarter more
// matrix instructions, and for heads wider than 64 its registers leave one wave per
// SIMD.  Steps, forward and backward: two samples of 8192 in documents, 32 and 8
// heads of 128: 2590 -> 2990 us (dQ 833 -> 1310), 3060 by going over the keys twice,
// x first, with two waves; 4 samples of 2048, 16 heads of 64: 248 -> 260, twice 297.
//
// e, which is small where it cancels, is taken as the sum of two bf16 values in its
// products, p where workgroups are small: with one each, errors were 1.5 times the
// outputs' own rounding, with two 1.25 (dQ 707 -> 833 us, dK and dV 1260 -> 1364).
//
// Bound by the vector unit's work on the scores (exponent, cap, e, its rounding)
// and the matrix instructions, which take turns: 32 samples of 128, 12 heads of 64:
// dQ 16, dK and dV 13 us.
//
// As in the forward pass, a block whose sums are not finite is formed again row
// by row, over visible pairs only.  Padding does not get there: rows that see nothing
// are taken as zeros, and tiles of queries repeat a row that counts in their place.
#pragma once

#include "attention_backward.hpp"

#include "attention_tile.hpp"

#include <type_traits>

namespace dpg {
namespace attn {
namespace {

constexpr int kGroup = 1024;             // tiles in a list

template <typename T, int DP, bool SMALL>
struct Shape {
    typedef Tile<T, DP> TL;
    static constexpr int NW = SMALL && TL::RB >= 384 ? 2 : 4;
    static constexpr int BN = SMALL || sizeof(T) == 4 ? 32 : 64;         // rows of a staged tile
    static constexpr int BR = SMALL ? 32 : 32 * NW;                      // rows (or keys) of a workgroup
    static constexpr int FN = BN / 32, THREADS = 64 * NW;
    static constexpr int HALF = BN * TL::RB, INFO = 2 * 256, STAGE = 2 * HALF + INFO;
    static constexpr int OUT_ROW = SMALL ? DP * 4 + 16 : TL::RB + 16;    // bytes of an output row in LDS
    static constexpr int STAGES = (SMALL ? NW : 1) * 2 * STAGE, OUTPUT = NW * 32 * OUT_ROW;
    static constexpr int LDS = STAGES > OUTPUT ? STAGES : OUTPUT;
};

// Ordered list of the tiles [t0, t1) that classify() does not skip: entries (tile - t0) << 2 | class; returns their number.
// Every thread of the workgroup takes part.
template <int THREADS, typename F>
__device__ __forceinline__ int tile_list(int t0, int t1, uint16_t *list, uint8_t *cls_of, int *counts, F &&classify)
{
    const int lane = threadIdx.x & 63;
    __syncthreads();
    for (int k = threadIdx.x; k < kGroup; k += THREADS) {
        const int cls = k < t1 - t0 ? classify(t0 + k) : kSkip;
        cls_of[k] = (uint8_t)cls;
        const unsigned long long some = __ballot(cls != kSkip);
        if (lane == 0) counts[k >> 6] = __popcll(some);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < kGroup; k += THREADS) {
        const int cls = cls_of[k];
        const unsigned long long some = __ballot(cls != kSkip);
        int at = __popcll(some & ((1ull << lane) - 1));
        for (int w = 0; w < k >> 6; ++w) at += counts[w];
        if (cls != kSkip) list[at] = (uint16_t)(k << 2 | cls);
    }
    int count = 0;
    for (int w = 0; w < kGroup / 64; ++w) count += counts[w];
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(count);
}

// range of docs[p0 .. p1], by one wave
__device__ __forceinline__ void wave_docs_range(const int32_t *docs, int p0, int p1, int lane, int &lo, int &hi)
{
    lo = 0x7fffffff;
    hi = -0x7fffffff - 1;
    for (int p = p0 + lane; p <= p1; p += 64) {
        const int d = docs[p];
        lo = d < lo ? d : lo;
        hi = d > hi ? d : hi;
    }
    for (int off = 32; off >= 1; off >>= 1) {
        const int l2 = __shfl_xor(lo, off, kWave), h2 = __shfl_xor(hi, off, kWave);
        lo = l2 < lo ? l2 : lo;
        hi = h2 > hi ? h2 : hi;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
}

// 32 output rows from LDS rows of LDT bytes (values of T); to(row): where the row lies, or NULL
template <typename T, int DP, int LDT, typename F>
__device__ __forceinline__ void store_rows(const char *L, int D, bool vec, int lane, F &&to)
{
    typedef Tile<T, DP> TL;
#pragma unroll 4
    for (int at = lane; at < 32 * TL::PIECES; at += kWave) {
        const int row = at / TL::PIECES, d = (at - row * TL::PIECES) * TL::N;
        T *o = d < D ? to(row) : nullptr;
        if (o == nullptr) continue;
        const T *x = reinterpret_cast<const T *>(L + row * LDT) + d;
        if (vec) *reinterpret_cast<u32x4_t *>(o + d) = *reinterpret_cast<const u32x4_t *>(x);
        else
#pragma unroll
            for (int e = 0; e < TL::N; ++e)
                if (d + e < D) o[d + e] = x[e];
    }
}

// The sums of a block of 32 columns, f * acc, to memory: a wave's own (LARGE), or the waves' sums added in wave order (SMALL,
// all waves take part).  Returns whether a value is not finite.
template <typename T, int DP, typename S, bool SMALL, typename F>
__device__ __forceinline__ bool put_block(char *smem, f32x16_t (&acc)[Tile<T, DP>::DB], float f, int D, bool vec, int lane, int wave,
                                          F &&to)
{
    constexpr int DB = Tile<T, DP>::DB;
    const int li = lane & 31, h = lane >> 5;
    char *L = smem + wave * 32 * S::OUT_ROW + li * S::OUT_ROW;
    bool bad = false;
    if constexpr (!SMALL) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float v = f * acc[d][e];
                bad = bad || not_finite(v);
                store_elem(reinterpret_cast<T *>(L) + 32 * d + 8 * (e >> 2) + 4 * h + (e & 3), v);
            }
        store_rows<T, DP, S::OUT_ROW>(smem + wave * 32 * S::OUT_ROW, D, vec, lane, to);
        return bad;
    } else {
        __syncthreads();
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4 *>(L + 4 * (32 * d + 2 * e + 4 * h)) =
                    make_float4(acc[d][e], acc[d][e + 1], acc[d][e + 2], acc[d][e + 3]);
        __syncthreads();
        for (int at = threadIdx.x; at < 32 * (DP / 4); at += S::THREADS) {
            const int row = at / (DP / 4), d = 4 * (at - row * (DP / 4));
            auto *o = d < D ? to(row) : nullptr;
            if (o == nullptr) continue;
            float v[4] = {};
#pragma unroll
            for (int w = 0; w < S::NW; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(smem + (w * 32 + row) * S::OUT_ROW + 4 * d);
                v[0] += x.x;
                v[1] += x.y;
                v[2] += x.z;
                v[3] += x.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] *= f;
                bad = bad || not_finite(v[e]);
                if (d + e < D) store_elem(o + d + e, v[e]);
            }
        }
        return bad;
    }
}

template <int DB>
__device__ __forceinline__ void zero(f32x16_t (&acc)[DB])
{
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = 0.0f;
}

// ---------------------------------------------------------------------------
// dQ
// ---------------------------------------------------------------------------
template <typename T, int DP, bool VEC, int MOD, bool SMALL>
__global__ __launch_bounds__((Shape<T, DP, SMALL>::THREADS), (SMALL || Tile<T, DP>::RB >= 192 ? 1 : 2)) void query_kernel(
    Call c, Grads gr, int tiles_m, bool vec_out)
{
    typedef Shape<T, DP, SMALL> S;
    typedef Tile<T, DP> TL;
    constexpr int BN = S::BN, FN = S::FN, DB = TL::DB, KS = TL::KS, NW = S::NW;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    __shared__ uint16_t list[kGroup];
    __shared__ uint8_t cls_of[kGroup];
    __shared__ int counts[kGroup / 64];

    const int lane = threadIdx.x & 63, li = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = c.N * c.Hk;
    int nk = (int)blockIdx.x % heads, tm = tiles_m - 1 - (int)blockIdx.x / heads;
    if constexpr (!SMALL)
        if (gr.row_order != nullptr) {
            const int e = gr.row_order[(int)blockIdx.x / c.Hk], of = e / tiles_m;
            nk = of * c.Hk + (int)blockIdx.x % c.Hk;
            tm = e - of * tiles_m;
        }
    const int n = nk / c.Hk, kv = nk - n * c.Hk;
    const Sample smp(c, n);
    const int M = c.Tq * c.G, r0 = tm * S::BR, rw = SMALL ? r0 : r0 + 32 * wave;
    const T *K = (const T *)c.K + (i64)n * c.Tk * c.ldk + (i64)kv * c.D;
    const T *V = (const T *)c.V + (i64)n * c.Tk * c.ldv + (i64)kv * c.D;

    const int r = rw + li, i = r / c.G, g = r - i * c.G;
    const bool row_ok = r < M;
    const int pos = smp.first + i;
    const bool seeing = row_ok && pos >= 0 && pos < smp.L;
    const int lim = seeing ? smp.end_for(pos) : 0;
    const int doc = seeing && smp.docs != nullptr ? smp.docs[pos] : -1;
    const int head = kv * c.G + (row_ok ? g : 0);
    const i64 row = (i64)n * c.Tq + (row_ok ? i : 0), info = ((i64)n * c.Hq + head) * gr.pad + (row_ok ? i : 0);
    u32x4_t qf[KS], df[KS];
    TL::load_row((const T *)c.Q + row * c.ldq + (i64)head * c.D, c.D, seeing, VEC, lane, qf);
    TL::load_row((const T *)gr.dO + row * c.ldo + (i64)head * c.D, c.D, seeing, VEC, lane, df);
    // lse in units of ln 2 (+inf where the query sees nothing: its weights are then 0) and delta, which dK and dV's launch reads
    float lse2 = INFINITY, delta = 0.0f;
    {
        u32x4_t of[KS];
        TL::load_row((const T *)gr.O + row * c.ldo + (i64)head * c.D, c.D, seeing, VEC, lane, of);
        const float l = gr.lse[((i64)n * c.Hq + head) * c.Tq + (row_ok ? i : 0)];
        if (seeing && l != -INFINITY) lse2 = l * kLog2e;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) delta += TL::dot(of[ks], df[ks]);
        delta += other_half(delta);
        if (lse2 == INFINITY) delta = 0.0f;
    }
    // sum of p (dO.V - delta): what delta lacks, as O is rounded (fp32: no more than the sums' own roundings, and left in dQ)
    float excess = 0.0f;
    constexpr bool BESIDE = TL::BF16;
    const Scores<T, MOD> score(c);
    const float slope2 = (MOD & kSlope) != 0 && c.slopes != nullptr ? c.slopes[head] * kLog2e : 0.0f;

    RowSpan span = span_of(smp, c.G, M, r0, S::BR);
    const int end = smp.end_for(span.pmax < span.pmin ? -1 : span.pmax), t1 = (end + BN - 1) / BN;
    if (smp.docs != nullptr) wave_docs_range(smp.docs, span.pmin, span.pmax, lane, span.dmin, span.dmax);

    typedef f32x16_t Sums[DB];
    Sums acc, beside;                                    // sums of e K and of p (1 - tanh^2) K
    zero(acc);
    if constexpr (BESIDE) zero(beside);
    const Stager<TL, T, BN, SMALL ? 1 : NW, VEC> stk(c.ldk, c.D, SMALL ? 0 : wave, lane), stv(c.ldv, c.D, SMALL ? 0 : wave, lane);
    char *mine = smem + (SMALL ? wave * 2 * S::STAGE : 0);
    const uint32_t lds0 = lds_addr(mine);
    const auto issue = [&](int t, int buf) __attribute__((always_inline)) {
        const i64 k0 = (i64)t * BN;
        const int left = (int)(end - k0);
        stk.issue(K + k0 * c.ldk, left, lds0 + buf * S::STAGE, mine + buf * S::STAGE);
        stv.issue(V + k0 * c.ldv, left, lds0 + buf * S::STAGE + S::HALF, mine + buf * S::STAGE + S::HALF);
    };
    const auto step = [&](const char *LK, const char *LV, int k0, int cls) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < FN; ++x) {
            f32x16_t s, e;
#pragma unroll
            for (int k = 0; k < 16; ++k) s[k] = e[k] = 0.0f;
            TL::template products<2>([&](int i, int ks) { return TL::rows(i == 0 ? LK : LV, 32 * x, ks, lane); },
                                     [&](int i, int ks) -> const u32x4_t & { return i == 0 ? qf[ks] : df[ks]; },
                                     [&](int i) -> f32x16_t & { return i == 0 ? s : e; });
            const auto key = [&](int k) __attribute__((always_inline)) { return k0 + 32 * x + 8 * (k >> 2) + 4 * h + (k & 3); };
            unsigned seen = 0;                           // bit k: the pair of row li and key(k) is visible
            if (cls != kFull) {
#pragma unroll
                for (int k = 0; k < 16; ++k) seen |= key(k) < lim ? 1u << k : 0u;
                if (cls == kDocs) {
                    // (all loads before the first comparison)
                    int d[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) d[k] = smp.docs[key(k) < end ? key(k) : end - 1];
#pragma unroll
                    for (int k = 0; k < 16; ++k) seen &= d[k] == doc && doc >= 0 ? ~0u : ~(1u << k);
                }
            }
            const auto weigh = [&](auto is_near, auto all) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    float bend;
                    const float p = __builtin_amdgcn_exp2f(score.template of<decltype(is_near)::value>(
                        s[k], lse2, slope2, __builtin_fabsf((float)(pos - key(k))), bend));
                    float g = p * (e[k] - delta);
                    if constexpr (!decltype(all)::value) g = (seen >> k & 1u) != 0 ? g : 0.0f;
                    excess += g;
                    if constexpr ((MOD & kCap) != 0) {
                        if constexpr (!decltype(all)::value) bend = (seen >> k & 1u) != 0 ? bend : 0.0f;
                        g *= bend;
                    }
                    e[k] = g;
                    if constexpr (BESIDE) {
                        s[k] = (MOD & kCap) != 0 ? p * bend : p;
                        if constexpr (!decltype(all)::value) s[k] = (seen >> k & 1u) != 0 ? s[k] : 0.0f;
                    }
                }
            };
            if (cls == kFull) {
                if (score.near(s)) weigh(std::true_type{}, std::true_type{});
                else weigh(std::false_type{}, std::true_type{});
            } else {
                if (score.near(s)) weigh(std::true_type{}, std::false_type{});
                else weigh(std::false_type{}, std::false_type{});
            }
            TL::template columns<1, 1>([&](int) { return LK + 32 * x * TL::RB; }, [&](int) -> const f32x16_t & { return e; },
                                       [&](int) -> Sums & { return acc; }, lane, [&](int step, int d, const bf16x8_t &a) __attribute__((always_inline)) {
                bf16x8_t b;
#pragma unroll
                for (int k = 0; k < 8; ++k) b[k] = (__bf16)s[8 * step + k];
                beside[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, beside[d], 0, 0, 0);
            });
        }
    };

    int base = 0;
    while (base < t1) {
        const bool docs = smp.docs != nullptr;
        const int stop = !docs || t1 - base <= kGroup ? t1 : base + kGroup;
        int count = stop - base;
        if (docs)
            count = tile_list<S::THREADS>(base, stop, list, cls_of, counts, [&](int t) {
                const int j0 = t * BN, j1 = j0 + BN < end ? j0 + BN : end;
                int lo, hi;
                docs_range(smp.docs, j0, j1, lo, hi);
                return meet(smp, span, j0, j0 + BN, lo, hi);
            });
        const auto entry = [&](int k, int &t, int &cls) __attribute__((always_inline)) {
            if (docs) {
                const int e = __builtin_amdgcn_readfirstlane(list[k]);
                t = base + (e >> 2);
                cls = e & 3;
            } else {
                t = base + k;
                cls = meet(smp, span, t * BN, t * BN + BN, 0, 0);
            }
        };
        int t, cls;
        constexpr int STEP = SMALL ? NW : 1;
        const int k0 = SMALL ? wave : 0;
        if (k0 < count) {
            entry(k0, t, cls);
            issue(t, 0);
            // (in blocks of 128 each buffer has code of its own, so that its places are constants of the LDS reads)
            const auto turn = [&](int k, int buf) __attribute__((always_inline)) {
                const int at = t * BN, now = cls;
                wait_loads();
                if constexpr (SMALL) bf16s::wait_lgkmcnt0();
                else lds_barrier();                     // this tile has landed, the one before is read
                if (k + STEP < count) {
                    entry(k + STEP, t, cls);
                    issue(t, buf ^ 1);
                }
                wave_together();
                step(mine + buf * S::STAGE, mine + buf * S::STAGE + S::HALF, at, now);
            };
            if constexpr (SMALL) {
                for (int k = k0, buf = 0; k < count; k += STEP, buf ^= 1) turn(k, buf);
            } else {
                for (int k = k0; k < count; k += 2) {
                    turn(k, 0);
                    if (k + 1 < count) turn(k + 1, 1);
                }
            }
        }
        if constexpr (!SMALL) lds_barrier();
        base = stop;
    }

    const auto to = [&](int k) __attribute__((always_inline)) -> T * {
        const int rr = rw + k, ik = rr / c.G;
        return rr < M ? (T *)gr.dQ + ((i64)n * c.Tq + ik) * c.ldq + (i64)(kv * c.G + rr - ik * c.G) * c.D : nullptr;
    };
    excess += other_half(excess);
    if constexpr (SMALL) {
        __syncthreads();                                 // all have read their tiles
        float *sums = reinterpret_cast<float *>(smem);
        if (h == 0) sums[wave * 32 + li] = excess;
        __syncthreads();
        excess = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) excess += sums[w * 32 + li];
    }
    if constexpr (BESIDE)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[d][k] = __builtin_fmaf(-excess, beside[d][k], acc[d][k]);
    if (row_ok && h == 0 && (!SMALL || wave == 0)) {
        gr.row_lse[info] = lse2;
        gr.row_delta[info] = delta + excess;
    }
    const bool bad = put_block<T, DP, S, SMALL>(smem, acc, c.scale, c.D, vec_out, lane, wave, to);
    wait_loads();                                        // the stores above come before those below
    if (SMALL ? __syncthreads_or(bad) : __any(bad))
        for (int k = SMALL ? wave : 0; k < 32 && rw + k < M; k += SMALL ? NW : 1) {
            const int ik = (rw + k) / c.G;
            backward_query_row<T>(c, n, kv * c.G + rw + k - ik * c.G, ik, (const T *)gr.O, gr.lse, (const T *)gr.dO, (T *)gr.dQ, nullptr);
        }
}

// ---------------------------------------------------------------------------
// dK and dV
// ---------------------------------------------------------------------------
// (Rows of 192 bytes or longer leave one wave per SIMD, by sums and operands of 260 registers and more.  Two samples of 8192 causal
// queries in documents, 32 and 8 heads of 128, capped scores, blocks in the order of positions, weights rounded once: 1717 us; dV and dK in launches of their own, two waves per SIMD and one product
// more, 813 + 1033; V's operands in LDS, two waves and some of K's in scratch memory, 2297.)
template <typename T, int DP, bool VEC, int MOD, bool SMALL>
__global__ __launch_bounds__((Shape<T, DP, SMALL>::THREADS), (SMALL || Tile<T, DP>::RB > 128 ? 1 : 2)) void key_kernel(
    Call c, Grads gr, bool vec_k, bool vec_v)
{
    typedef Shape<T, DP, SMALL> S;
    typedef Tile<T, DP> TL;
    constexpr int BN = S::BN, FN = S::FN, DB = TL::DB, KS = TL::KS, NW = S::NW;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    __shared__ uint16_t list[kGroup];
    __shared__ uint8_t cls_of[kGroup];
    __shared__ int counts[kGroup / 64];

    const int lane = threadIdx.x & 63, li = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = c.N * c.Hk;
    // first keys first: with a causal mask they have most queries
    const int split = SMALL ? (int)blockIdx.x % gr.splits : 0, at_block = SMALL ? (int)blockIdx.x / gr.splits : (int)blockIdx.x;
    int nk = at_block % heads, tk = at_block / heads;
    if constexpr (!SMALL)
        if (gr.key_order != nullptr) {
            const int blocks = (c.Tk + S::BR - 1) / S::BR, e = gr.key_order[at_block / c.Hk], of = e / blocks;
            nk = of * c.Hk + at_block % c.Hk;
            tk = e - of * blocks;
        }
    const int n = nk / c.Hk, kv = nk - n * c.Hk;
    const Sample smp(c, n);
    const int j0 = tk * S::BR, jw = SMALL ? j0 : j0 + 32 * wave;
    const T *Q = (const T *)c.Q + (i64)n * c.Tq * c.ldq + (i64)kv * c.G * c.D;
    const T *dO = (const T *)gr.dO + (i64)n * c.Tq * c.ldo + (i64)kv * c.G * c.D;
    const float *row_lse = gr.row_lse + ((i64)n * c.Hq + kv * c.G) * gr.pad;
    const float *row_delta = gr.row_delta + ((i64)n * c.Hq + kv * c.G) * gr.pad;

    const int j = jw + li;                               // this lane's key
    const bool key_ok = j < smp.L;
    const i64 krow = (i64)n * c.Tk + (key_ok ? j : 0);
    u32x4_t kf[KS], vf[KS];
    TL::load_row((const T *)c.K + krow * c.ldk + (i64)kv * c.D, c.D, key_ok, VEC, lane, kf);
    TL::load_row((const T *)c.V + krow * c.ldv + (i64)kv * c.D, c.D, key_ok, VEC, lane, vf);
    // queries at positions from .. L - 1 see it
    const int from = !key_ok ? 1 << 30 : !smp.causal || j < smp.prefix ? 0 : j;
    const int doc = key_ok && smp.docs != nullptr ? smp.docs[j] : -1;
    const Scores<T, MOD> score(c);

    // the block's keys, and the queries that may see one of them: [i0, i1)
    const int end = j0 + S::BR < smp.L ? j0 + S::BR : smp.L;
    int i0 = -smp.first, i1 = smp.L - smp.first;
    if (smp.causal && j0 >= smp.prefix) i0 = j0 - smp.first;
    i0 = i0 > 0 ? i0 : 0;
    i1 = i1 < c.Tq ? i1 : c.Tq;
    int kd0 = 0, kd1 = 0;
    if (j0 < smp.L && smp.docs != nullptr) wave_docs_range(smp.docs, j0, end - 1, lane, kd0, kd1);
    const int t0 = i0 / BN, t1 = j0 < smp.L && i0 < i1 ? (i1 + BN - 1) / BN : t0;

    typedef f32x16_t Sums[DB];
    Sums ak, av;
    zero(ak);
    zero(av);
    const Stager<TL, T, BN, SMALL ? 1 : NW, VEC> stq(c.ldq, c.D, SMALL ? 0 : wave, lane), std(c.ldo, c.D, SMALL ? 0 : wave, lane);
    char *mine = smem + (SMALL ? wave * 2 * S::STAGE : 0);
    const uint32_t lds0 = lds_addr(mine);
    const auto issue = [&](int t, int g, int buf) __attribute__((always_inline)) {
        const int q0 = t * BN;
        const uint32_t L = lds0 + buf * S::STAGE;
        stq.issue(Q + (i64)q0 * c.ldq + (i64)g * c.D, i1 - q0, L, mine + buf * S::STAGE, i0 - q0);
        std.issue(dO + (i64)q0 * c.ldo + (i64)g * c.D, i1 - q0, L + S::HALF, mine + buf * S::STAGE + S::HALF, i0 - q0);
        // 64 floats each, inside the padded rows: q0 is a multiple of BN, a short tile's are read twice
        if (SMALL || wave == 0) {
            const uint32_t off = 4u * (uint32_t)(lane & (BN - 1));
            dma4_off(row_lse + (i64)g * gr.pad + q0, off, L + 2 * S::HALF);
            dma4_off(row_delta + (i64)g * gr.pad + q0, off, L + 2 * S::HALF + 256);
        }
    };
    const auto step = [&](const char *L, int q0, int g, int cls) __attribute__((always_inline)) {
        const char *LQ = L, *LD = L + S::HALF;
        const float slope2 = (MOD & kSlope) != 0 && c.slopes != nullptr ? c.slopes[kv * c.G + g] * kLog2e : 0.0f;
#pragma unroll
        for (int x = 0; x < FN; ++x) {
            f32x16_t s, e;
#pragma unroll
            for (int k = 0; k < 16; ++k) s[k] = e[k] = 0.0f;
            TL::template products<2>([&](int i, int ks) { return TL::rows(i == 0 ? LQ : LD, 32 * x, ks, lane); },
                                                 [&](int i, int ks) -> const u32x4_t & { return i == 0 ? kf[ks] : vf[ks]; },
                                                 [&](int i) -> f32x16_t & { return i == 0 ? s : e; });
            const auto place = [&](int k) __attribute__((always_inline)) { return 32 * x + 8 * (k >> 2) + 4 * h + (k & 3); };
            const auto weigh = [&](auto is_near) __attribute__((always_inline)) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float4 l4 = *reinterpret_cast<const float4 *>(L + 2 * S::HALF + 4 * (32 * x + 8 * b + 4 * h));
                    const float4 d4 = *reinterpret_cast<const float4 *>(L + 2 * S::HALF + 256 + 4 * (32 * x + 8 * b + 4 * h));
                    const float lse2[4] = {l4.x, l4.y, l4.z, l4.w}, delta[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int k = 4 * b + w;
                        float bend;
                        s[k] = __builtin_amdgcn_exp2f(score.template of<decltype(is_near)::value>(
                            s[k], lse2[w], slope2, __builtin_fabsf((float)(smp.first + q0 + place(k) - j)), bend));
                        e[k] = s[k] * (e[k] - delta[w]);
                        if constexpr ((MOD & kCap) != 0) e[k] *= bend;
                    }
                }
            };
            if (score.near(s)) weigh(std::true_type{});
            else weigh(std::false_type{});
            if (cls != kFull) {
                const int lo = from - smp.first - q0, hi = (smp.L - smp.first < c.Tq ? smp.L - smp.first : c.Tq) - q0;
                const auto hide = [&](auto &&seen) __attribute__((always_inline)) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const bool see = seen(k);
                        s[k] = see ? s[k] : 0.0f;
                        e[k] = see ? e[k] : 0.0f;
                    }
                };
                hide([&](int k) { return place(k) >= lo && place(k) < hi; });
                if (cls == kDocs) {
                    // (all loads before the first comparison)
                    int d[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        int p = smp.first + q0 + place(k);
                        p = p > 0 ? p : 0;
                        d[k] = smp.docs[p < smp.L ? p : smp.L - 1];
                    }
                    hide([&](int k) { return d[k] == doc && doc >= 0; });
                }
            }
            const char *LX = L + 32 * x * TL::RB;
            TL::template columns<2, SMALL ? 3 : 2>([&](int i) { return i == 0 ? LX + S::HALF : LX; },
                                    [&](int i) -> const f32x16_t & { return i == 0 ? s : e; },
                                    [&](int i) -> Sums & { return i == 0 ? av : ak; }, lane);
        }
    };

    int base = t0;
    while (base < t1) {
        const bool docs = smp.docs != nullptr;
        const int stop = !docs || t1 - base <= kGroup ? t1 : base + kGroup;
        const auto class_of = [&](int t, bool with_docs) __attribute__((always_inline)) {
            RowSpan span = span_of(smp, 1, c.Tq, t * BN, BN);
            if (with_docs) docs_range(smp.docs, span.pmin, span.pmax + 1, span.dmin, span.dmax);
            return meet(smp, span, j0, j0 + S::BR, kd0, kd1);
        };
        int count = stop - base;
        if (docs)
            count = tile_list<S::THREADS>(base, stop, list, cls_of, counts, [&](int t) { return class_of(t, true); });
        // the heads one after another, each over the tiles; this split's part of them
        const int whole = count * c.G, all = SMALL ? (int)((i64)whole * (split + 1) / gr.splits) : whole;
        const auto entry = [&](int k, int &t, int &g, int &cls) __attribute__((always_inline)) {
            g = k / count;
            if (docs) {
                const int e = __builtin_amdgcn_readfirstlane(list[k - g * count]);
                t = base + (e >> 2);
                cls = e & 3;
            } else {
                t = base + k - g * count;
                cls = class_of(t, false);
            }
        };
        int t, g, cls;
        constexpr int STEP = SMALL ? NW : 1;
        const int k0 = SMALL ? (int)((i64)whole * split / gr.splits) + wave : 0;
        if (k0 < all) {
            entry(k0, t, g, cls);
            issue(t, g, 0);
            const auto turn = [&](int k, int buf) __attribute__((always_inline)) {
                const int at = t * BN, head = g, now = cls;
                wait_loads();
                if constexpr (SMALL) bf16s::wait_lgkmcnt0();
                else lds_barrier();                     // this tile has landed, the one before is read
                if (k + STEP < all) {
                    entry(k + STEP, t, g, cls);
                    issue(t, g, buf ^ 1);
                }
                wave_together();
                step(mine + buf * S::STAGE, at, head, now);
            };
            if constexpr (SMALL) {
                for (int k = k0, buf = 0; k < all; k += STEP, buf ^= 1) turn(k, buf);
            } else {
                for (int k = k0; k < all; k += 2) {
                    turn(k, 0);
                    if (k + 1 < all) turn(k + 1, 1);
                }
            }
        }
        if constexpr (!SMALL) lds_barrier();
        base = stop;
    }

    if constexpr (SMALL)
        if (gr.splits > 1) {
            const auto part_of = [&](int which, int k) __attribute__((always_inline)) -> float * {
                return jw + k < c.Tk ? gr.part + (((i64)split * heads + nk) * c.Tk + jw + k) * 2 * c.D + which * c.D : nullptr;
            };
            put_block<T, DP, S, SMALL>(smem, ak, c.scale, c.D, false, lane, wave, [&](int k) { return part_of(0, k); });
            put_block<T, DP, S, SMALL>(smem, av, 1.0f, c.D, false, lane, wave, [&](int k) { return part_of(1, k); });
            return;
        }
    const auto row_of = [&](void *p, i64 ld, int k) __attribute__((always_inline)) -> T * {
        return jw + k < c.Tk ? (T *)p + ((i64)n * c.Tk + jw + k) * ld + (i64)kv * c.D : nullptr;
    };
    bool bad = put_block<T, DP, S, SMALL>(smem, ak, c.scale, c.D, vec_k, lane, wave, [&](int k) { return row_of(gr.dK, c.ldk, k); });
    bad |= put_block<T, DP, S, SMALL>(smem, av, 1.0f, c.D, vec_v, lane, wave, [&](int k) { return row_of(gr.dV, c.ldv, k); });
    wait_loads();                                        // the stores above come before those below
    if (SMALL ? __syncthreads_or(bad) : __any(bad))
        for (int k = SMALL ? wave : 0; k < 32 && jw + k < c.Tk; k += SMALL ? NW : 1)
            backward_key_row<T>(c, n, kv, jw + k, gr.lse, gr.row_delta, gr.pad, (const T *)gr.dO, (T *)gr.dK, (T *)gr.dV);
}

// A wave adds a key's sums over the splits, in their order.
template <typename T>
__global__ __launch_bounds__(256) void key_join_kernel(Call c, Grads gr)
{
    constexpr int PER = kTileD / kWave;
    const i64 rows = (i64)c.N * c.Hk * c.Tk, r = (i64)blockIdx.x * 4 + threadIdx.x / kWave;
    if (r >= rows) return;
    const int lane = threadIdx.x & (kWave - 1), nk = (int)(r / c.Tk), j = (int)(r - (i64)nk * c.Tk), n = nk / c.Hk, kv = nk - n * c.Hk;
    float v[2][PER] = {};
    bool bad = false;
#pragma unroll 4
    for (int s = 0; s < gr.splits; ++s)
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (lane + kWave * k < c.D) v[w][k] += gr.part[((s * rows + r) * 2 + w) * c.D + lane + kWave * k];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int k = 0; k < PER; ++k) bad = bad || not_finite(v[w][k]);
    if (__any(bad)) {
        backward_key_row<T>(c, n, kv, j, gr.lse, gr.row_delta, gr.pad, (const T *)gr.dO, (T *)gr.dK, (T *)gr.dV);
        return;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (lane + kWave * k < c.D) {
            store_elem((T *)gr.dK + ((i64)n * c.Tk + j) * c.ldk + (i64)kv * c.D + lane + kWave * k, v[0][k]);
            store_elem((T *)gr.dV + ((i64)n * c.Tk + j) * c.ldv + (i64)kv * c.D + lane + kWave * k, v[1][k]);
        }
}

template <typename T, int DP, bool VEC, int MOD>
void launch(const Call &c, const Grads &g, hipStream_t stream)
{
    constexpr int N = 16 / sizeof(T);
    const i64 heads = (i64)c.N * c.Hk, M = (i64)c.Tq * c.G;
    const auto wide = [&](const void *p, i64 ld) __attribute__((always_inline)) { return c.D % N == 0 && ld % N == 0 && aligned(p, 16); };
    if (M > 0) {
        const int tiles = (int)ceil_div(M, g.small_q ? 32 : 128);
        if (g.small_q)
            query_kernel<T, DP, VEC, MOD, true><<<(unsigned)(heads * tiles), Shape<T, DP, true>::THREADS, 0, stream>>>(
                c, g, tiles, wide(g.dQ, c.ldq));
        else
            query_kernel<T, DP, VEC, MOD, false><<<(unsigned)(heads * tiles), Shape<T, DP, false>::THREADS, 0, stream>>>(
                c, g, tiles, wide(g.dQ, c.ldq));
    }
    if (c.Tk > 0) {
        const unsigned blocks = (unsigned)(heads * ceil_div(c.Tk, g.small_k ? 32 : 128) * (g.small_k ? g.splits : 1));
        const bool vk = wide(g.dK, c.ldk), vv = wide(g.dV, c.ldv);
        if (g.small_k) key_kernel<T, DP, VEC, MOD, true><<<blocks, Shape<T, DP, true>::THREADS, 0, stream>>>(c, g, vk, vv);
        else key_kernel<T, DP, VEC, MOD, false><<<blocks, Shape<T, DP, false>::THREADS, 0, stream>>>(c, g, vk, vv);
        if (g.small_k && g.splits > 1)
            key_join_kernel<T><<<(unsigned)ceil_div(heads * c.Tk, 4), 256, 0, stream>>>(c, g);
    }
}

template <typename T, int DP>
void by_kind(const Call &c, const Grads &g, hipStream_t stream)
{
    constexpr int N = 16 / sizeof(T);
    const bool vec = c.D % N == 0 && c.ldq % N == 0 && c.ldk % N == 0 && c.ldv % N == 0 && c.ldo % N == 0 && aligned(c.Q, 16) &&
                     aligned(c.K, 16) && aligned(c.V, 16) && aligned(g.O, 16) && aligned(g.dO, 16);
    const int mod = c.scale <= 0.0f ? kBoth : (c.cap > 0.0f ? kCap : kPlain) | (c.slopes != nullptr ? kSlope : kPlain);
    if (!vec) launch<T, DP, false, kBoth>(c, g, stream);
    else if (mod == kPlain) launch<T, DP, true, kPlain>(c, g, stream);
    else if (mod == kCap) launch<T, DP, true, kCap>(c, g, stream);
    else if (mod == kSlope) launch<T, DP, true, kSlope>(c, g, stream);
    else launch<T, DP, true, kBoth>(c, g, stream);
}

template <typename T>
dp_status tiles_of(const Call &c, const Grads &g, hipStream_t stream)
{
    if (c.D <= 32) by_kind<T, 32>(c, g, stream);
    else if (c.D <= 64) by_kind<T, 64>(c, g, stream);
    else if (c.D <= 96) by_kind<T, 96>(c, g, stream);
    else by_kind<T, 128>(c, g, stream);
    return launch_status();
}

}  // namespace
}  // namespace attn
}  // namespace dpg
