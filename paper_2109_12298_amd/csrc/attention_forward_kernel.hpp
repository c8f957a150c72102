// Attention forward: one pass over the keys with the running maximum and sum of
// the softmax.
//
// A wave has 32 rows (attention_tile.hpp) and forms scores as keys x rows, so
// that a row's scores lie in two lanes: maximum and sum need one exchange, and
// the weights go to the second product from the registers they were formed in.
// The accumulators are multiplied anew only where a row's maximum grows by more
// than 2^8: weights are then at most 2^8, which costs neither fp32 sums nor
// bf16 weights a bit.
//
// Two shapes.  Blocks of 128 rows (four waves) share tiles of keys, two stages
// deep, where there are blocks enough to fill the card.  Else 32 rows are one
// workgroup whose waves take different tiles of keys, and with few rows several
// workgroups split a sample's keys, each a run of its own length L / splits:
// their sums are joined by a second launch, in the order of the runs.
//
// With bf16 values the weights are rounded to bf16 for their product, which turns the
// outputs' own rounding (a relative error of 1.7e-3 in the mean square) into 2.0 to
// 2.4e-3; where workgroups are small, which memory or latency bounds, they are the
// sum of two bf16 values instead.
//
// Two prompts of 4096, 32 and 8 heads of 128, bf16: 276 to 290 us, 950 TFLOP/s (209
// at a large product's rate): softmax on the vector unit and matrix instructions of
// one SIMD's two waves overlap in part.  One query over 4096 keys: 6 us and the join's
// 4; 32 queries over up to 8192 keys each: 117 us, 5.2 TB/s of K and V.
//
// Hidden pairs have weight 0 by selection; an infinity or NaN in their values
// would still turn 0 into NaN in the product, so a block whose sums are not
// finite is formed again row by row, over visible pairs only; so is one whose sums
// vanish, as they may for scores past 2^29 (inverse_sum).
#pragma once

#include "attention_forward.hpp"

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
    static constexpr int BN = SMALL || sizeof(T) == 4 ? 32 : 64;         // keys in a tile
    static constexpr int BR = SMALL ? 32 : 32 * NW;                      // rows of a workgroup
    static constexpr int FN = BN / 32, THREADS = 64 * NW;
    static constexpr int HALF = BN * TL::RB, STAGE = 2 * HALF;           // K, then V
    static constexpr int OUT_ROW = SMALL ? DP * 4 + 16 : TL::RB + 16;    // bytes of an output row in LDS
    static constexpr int STAGES = (SMALL ? NW : 2) * STAGE, OUTPUT = NW * 32 * OUT_ROW;
    static constexpr int LDS = STAGES > OUTPUT ? STAGES : OUTPUT;
};

// 32 output rows from LDS rows of LDT bytes (values of T)
template <typename T, int DP, int LDT>
__device__ __forceinline__ void store_rows(const Call &c, const char *L, T *O, int n, int kv, int r0, int M, bool vec, int lane,
                                           i64 ld)
{
    typedef Tile<T, DP> TL;
#pragma unroll 4
    for (int at = lane; at < 32 * TL::PIECES; at += kWave) {
        const int row = at / TL::PIECES, d = (at - row * TL::PIECES) * TL::N, r = r0 + row;
        if (r >= M || d >= c.D) continue;
        const int i = r / c.G, g = r - i * c.G;
        T *o = O + ((i64)n * c.Tq + i) * ld + (i64)(kv * c.G + g) * c.D + d;
        const T *x = reinterpret_cast<const T *>(L + row * LDT) + d;
        if (vec) *reinterpret_cast<u32x4_t *>(o) = *reinterpret_cast<const u32x4_t *>(x);
        else
#pragma unroll
            for (int e = 0; e < TL::N; ++e)
                if (d + e < c.D) o[e] = x[e];
    }
}

template <typename T, int DP, bool VEC, int MOD, bool SMALL>
__global__ __launch_bounds__((Shape<T, DP, SMALL>::THREADS), (SMALL || Tile<T, DP>::RB >= 512 ? 1 : 2)) void forward_kernel(Call c, ForwardOut out, int tiles_m,
                                                                                              bool vec_out)
{
    typedef Shape<T, DP, SMALL> S;
    typedef Tile<T, DP> TL;
    constexpr int BN = S::BN, FN = S::FN, DB = TL::DB, KS = TL::KS, NW = S::NW;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
    __shared__ uint16_t list[kGroup];
    __shared__ uint8_t cls_of[kGroup];
    __shared__ int counts[kGroup / 64], doc_lo, doc_hi;
    __shared__ float join[2][NW][32];

    const int lane = threadIdx.x & 63, li = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // key heads fastest (consecutive blocks go to different XCDs, blocks of one key head to the same where the heads are a
    // multiple of 8), rows from the last block on: with a causal mask it has most keys
    const int heads = c.N * c.Hk;
    int b = (int)blockIdx.x, split = 0;
    if constexpr (SMALL) {
        split = b % out.splits;
        b /= out.splits;
    }
    int nk = b % heads, tm = tiles_m - 1 - b / heads;
    if constexpr (!SMALL)
        if (out.order != nullptr) {
            const int e = out.order[b / c.Hk], of = e / tiles_m;
            nk = of * c.Hk + b % c.Hk;
            tm = e - of * tiles_m;
        }
    const int n = nk / c.Hk, kv = nk - n * c.Hk;
    const Sample smp(c, n);
    const int M = c.Tq * c.G, r0 = tm * S::BR, rw = SMALL ? r0 : r0 + 32 * wave;
    const T *K = (const T *)c.K + (i64)n * c.Tk * c.ldk + (i64)kv * c.D;
    const T *V = (const T *)c.V + (i64)n * c.Tk * c.ldv + (i64)kv * c.D;

    // this lane's row
    const int r = rw + li, i = r / c.G, g = r - i * c.G;
    const bool row_ok = r < M;
    const int pos = smp.first + i;
    const bool seeing = row_ok && pos >= 0 && pos < smp.L;
    const int lim = seeing ? smp.end_for(pos) : 0;
    const int doc = seeing && smp.docs != nullptr ? smp.docs[pos] : -1;
    const int head = kv * c.G + (row_ok ? g : 0);
    u32x4_t qf[KS];
    TL::load_row((const T *)c.Q + ((i64)n * c.Tq + (row_ok ? i : 0)) * c.ldq + (i64)head * c.D, c.D, seeing, VEC, lane, qf);
    const Scores<T, MOD> score(c);
    const float slope2 = (MOD & kSlope) != 0 && c.slopes != nullptr ? c.slopes[head] * kLog2e : 0.0f;

    RowSpan span = span_of(smp, c.G, M, r0, S::BR);
    // keys of this workgroup
    const int end = smp.end_for(span.pmax < span.pmin ? -1 : span.pmax);
    int t0 = 0, t1 = (end + BN - 1) / BN;
    if constexpr (SMALL) {
        if (out.splits > 1) {
            const int per = (int)(((i64)smp.L + (i64)out.splits * BN - 1) / ((i64)out.splits * BN));
            t0 = split * per;
            t1 = t1 < t0 + per ? t1 : t0 + per;
        }
    }
    if (smp.docs != nullptr && t0 < t1) {
        // the rows' documents' range
        if (threadIdx.x < 64) {
            int lo = 0x7fffffff, hi = -0x7fffffff - 1;
            for (int p = span.pmin + lane; p <= span.pmax; p += 64) {
                const int d = smp.docs[p];
                lo = d < lo ? d : lo;
                hi = d > hi ? d : hi;
            }
            for (int off = 32; off >= 1; off >>= 1) {
                const int l2 = __shfl_xor(lo, off, kWave), h2 = __shfl_xor(hi, off, kWave);
                lo = l2 < lo ? l2 : lo;
                hi = h2 > hi ? h2 : hi;
            }
            if (lane == 0) {
                doc_lo = lo;
                doc_hi = hi;
            }
        }
        __syncthreads();
        span.dmin = __builtin_amdgcn_readfirstlane(doc_lo);
        span.dmax = __builtin_amdgcn_readfirstlane(doc_hi);
    }

    f32x16_t acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = 0.0f;
    float top = -INFINITY, sum = 0.0f;

    const Stager<TL, T, BN, SMALL ? 1 : NW, VEC> stk(c.ldk, c.D, SMALL ? 0 : wave, lane), stv(c.ldv, c.D, SMALL ? 0 : wave, lane);
    char *mine = smem + (SMALL ? wave * S::STAGE : 0);
    const uint32_t lds0 = lds_addr(mine);
    const auto issue_k = [&](int t, int buf) __attribute__((always_inline)) {
        const i64 k0 = (i64)t * BN;
        stk.issue(K + k0 * c.ldk, (int)(end - k0), lds0 + buf * S::STAGE, mine + buf * S::STAGE);
    };
    const auto issue_v = [&](int t, int buf) __attribute__((always_inline)) {
        const i64 k0 = (i64)t * BN;
        stv.issue(V + k0 * c.ldv, (int)(end - k0), lds0 + buf * S::STAGE + S::HALF, mine + buf * S::STAGE + S::HALF);
    };
    f32x16_t s[FN];
    const auto scores = [&](const char *LK) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < FN; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[x][e] = 0.0f;
        TL::template products<FN>([&](int x, int ks) { return TL::rows(LK, 32 * x, ks, lane); },
                                  [&](int, int ks) -> const u32x4_t & { return qf[ks]; },
                                  [&](int x) -> f32x16_t & { return s[x]; });
    };
    // scores to weights, running maximum and sum
    const auto soften = [&](int k0, int cls) __attribute__((always_inline)) {
        const auto key = [&](int x, int e) __attribute__((always_inline)) { return k0 + 32 * x + 8 * (e >> 2) + 4 * h + (e & 3); };
        const auto far = [&](int x, int e) __attribute__((always_inline)) { return __builtin_fabsf((float)(pos - key(x, e))); };
        const auto each = [&](auto &&f) __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < FN; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[x][e] = f(x, e, s[x][e]);
        };
        const auto hide = [&](float with) __attribute__((always_inline)) {
            each([&](int x, int e, float v) { return key(x, e) < lim ? v : with; });
            if (cls == kDocs) {
                // (all loads before the first comparison)
                int d[FN][16];
#pragma unroll
                for (int x = 0; x < FN; ++x)
#pragma unroll
                    for (int e = 0; e < 16; ++e) d[x][e] = smp.docs[key(x, e) < end ? key(x, e) : end - 1];
                each([&](int x, int e, float v) { return d[x][e] == doc && doc >= 0 ? v : with; });
            }
        };
        float unused;
        bool near = MOD == kCap;
        if constexpr (MOD == kCap)
#pragma unroll
            for (int x = 0; x < FN; ++x) near = near && score.near(s[x]);
        if constexpr (MOD >= kSlope) each([&](int x, int e, float v) { return score.template of<false>(v, 0.0f, slope2, far(x, e), unused); });
        if (cls != kFull) hide(-INFINITY);
        float t = s[0][0];
#pragma unroll
        for (int x = 0; x < FN; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) t = fmaxf(t, s[x][e]);
        t = fmaxf(t, other_half(t));
        if constexpr (MOD == kPlain) t *= score.scale2;
        if constexpr (MOD == kCap) t = t == -INFINITY ? t : score.cap2 * tanh_for<T>(score.y_scale * t, unused);
        if (__any(t > top + 8.0f)) {
            const float was = top;
            top = fmaxf(top, t);
            const float f = __builtin_amdgcn_exp2f(was - (top == -INFINITY ? 0.0f : top));
            sum *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[d][e] *= f;
        }
        const float base = top == -INFINITY ? 0.0f : top;
        const auto weigh = [&](auto is_near) __attribute__((always_inline)) {
            each([&](int, int, float v) {
                return __builtin_amdgcn_exp2f(
                    MOD >= kSlope ? v - base : score.template of<decltype(is_near)::value>(v, base, 0.0f, 0.0f, unused));
            });
        };
        if constexpr (MOD == kCap) {
            if (near) weigh(std::true_type{});
            else weigh(std::false_type{});
            if (cls != kFull) hide(0.0f);               // (tanh of a hidden score, -inf, is -1, and the polynomial's may be NaN)
        } else {
            weigh(std::false_type{});
        }
#pragma unroll
        for (int x = 0; x < FN; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum += s[x][e];
    };
    const auto values = [&](const char *LV) __attribute__((always_inline)) {
        typedef f32x16_t Sums[DB];
        TL::template columns<FN, SMALL ? (1u << FN) - 1 : 0>([&](int x) { return LV + 32 * x * TL::RB; }, [&](int x) -> const f32x16_t & { return s[x]; },
                                 [&](int) -> Sums & { return acc; }, lane);
    };

    for (int base = t0; base < t1; base += kGroup) {
        int count = t1 - base;
        if (smp.docs != nullptr) {
            count = count < kGroup ? count : kGroup;
            __syncthreads();
            for (int k = threadIdx.x; k < kGroup; k += S::THREADS) {
                int cls = kSkip;
                if (k < count) {
                    const int j0 = (base + k) * BN, j1 = j0 + BN < end ? j0 + BN : end;
                    int lo, hi;
                    docs_range(smp.docs, j0, j1, lo, hi);
                    cls = meet(smp, span, j0, j0 + BN, lo, hi);
                }
                cls_of[k] = (uint8_t)cls;
                const unsigned long long some = __ballot(cls != kSkip);
                if (lane == 0) counts[k >> 6] = __popcll(some);
            }
            __syncthreads();
            for (int k = threadIdx.x; k < kGroup; k += S::THREADS) {
                const int cls = cls_of[k];
                const unsigned long long some = __ballot(cls != kSkip);
                int at = __popcll(some & ((1ull << lane) - 1));
                for (int w = 0; w < k >> 6; ++w) at += counts[w];
                if (cls != kSkip) list[at] = (uint16_t)(k << 2 | cls);
            }
            count = 0;
            for (int w = 0; w < kGroup / 64; ++w) count += counts[w];
            count = __builtin_amdgcn_readfirstlane(count);
            __syncthreads();
        } else {
            base = t1;                                  // one group
        }
        const int first = smp.docs != nullptr ? base : t0;
        const auto entry = [&](int k, int &t, int &cls) __attribute__((always_inline)) {
            if (smp.docs != nullptr) {
                const int e = __builtin_amdgcn_readfirstlane(list[k]);
                t = first + (e >> 2);
                cls = e & 3;
            } else {
                t = first + k;
                cls = meet(smp, span, t * BN, t * BN + BN, 0, 0);
            }
        };
        int t, cls;
        if constexpr (SMALL) {
            // a wave's own tiles, in its own buffers: K's takes the next tile once the scores are formed, V's once the sums are
            if (wave < count) {
                entry(wave, t, cls);
                issue_k(t, 0);
                issue_v(t, 0);
                for (int k = wave; k < count; k += NW) {
                    const int k0 = t * BN, now = cls;
                    const bool more = k + NW < count;
                    if constexpr (VEC) bf16s::wait_vmcnt<decltype(stv)::LOADS>();
                    bf16s::wait_lgkmcnt0();
                    wave_together();
                    scores(mine);
                    bf16s::wait_lgkmcnt0();
                    if (more) {
                        entry(k + NW, t, cls);
                        issue_k(t, 0);
                    }
                    soften(k0, now);
                    if constexpr (VEC) {
                        if (more) bf16s::wait_vmcnt<decltype(stk)::LOADS>();
                        else wait_loads();
                    }
                    bf16s::wait_lgkmcnt0();
                    wave_together();
                    values(mine + S::HALF);
                    bf16s::wait_lgkmcnt0();
                    if (more) issue_v(t, 0);
                }
            }
        } else {
            if (count > 0) {
                entry(0, t, cls);
                issue_k(t, 0);
                issue_v(t, 0);
                // (each buffer has code of its own, so that its places are constants of the LDS reads)
                const auto turn = [&](int k, int buf) __attribute__((always_inline)) {
                    const int k0 = t * BN, now = cls;
                    wait_loads();
                    lds_barrier();                      // this tile has landed, the one before is read
                    if (k + 1 < count) {
                        entry(k + 1, t, cls);
                        issue_k(t, buf ^ 1);
                        issue_v(t, buf ^ 1);
                    }
                    const char *L = smem + buf * S::STAGE;
                    wave_together();
                    scores(L);
                    soften(k0, now);
                    values(L + S::HALF);
                };
                for (int k = 0; k < count; k += 2) {
                    turn(k, 0);
                    if (k + 1 < count) turn(k + 1, 1);
                }
            }
            lds_barrier();
        }
    }

    sum += other_half(sum);
    if constexpr (!SMALL) {
        const float inv = inverse_sum(sum, top);
        bool bad = not_finite(sum) || not_finite(inv);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                acc[d][e] *= inv;
                bad = bad || not_finite(acc[d][e]);
            }
        if (__any(bad && row_ok)) {
            for (int k = 0; k < 32 && rw + k < M; ++k) {
                const int ik = (rw + k) / c.G;
                forward_row<T>(c, n, kv * c.G + (rw + k) - ik * c.G, ik, (T *)out.O, out.lse);
            }
            return;
        }
        if (out.lse != nullptr && row_ok && h == 0)
            out.lse[((i64)n * c.Hq + head) * c.Tq + i] = sum == 0.0f ? -INFINITY : top * kLn2 + logf(sum);
        char *L = smem + wave * 32 * S::OUT_ROW;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                T *o = reinterpret_cast<T *>(L + li * S::OUT_ROW) + 32 * d + 2 * e + 4 * h;
#pragma unroll
                for (int x = 0; x < 4; ++x) store_elem(o + x, acc[d][e + x]);
            }
        store_rows<T, DP, S::OUT_ROW>(c, L, (T *)out.O, n, kv, rw, M, vec_out, lane, c.ldo);
    } else {
        // the waves' sums to one maximum, added in wave order
        __syncthreads();                                 // all have read their tiles
        if (h == 0) join[0][wave][li] = top;
        if (h == 0) join[1][wave][li] = sum;
        __syncthreads();
        float all = -INFINITY, total = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) all = fmaxf(all, join[0][w][li]);
        const float base = all == -INFINITY ? 0.0f : all;
#pragma unroll
        for (int w = 0; w < NW; ++w) total += join[1][w][li] * __builtin_amdgcn_exp2f(join[0][w][li] - base);
        const float f = __builtin_amdgcn_exp2f(top - base);
        char *L = smem + wave * 32 * S::OUT_ROW;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4 *>(L + li * S::OUT_ROW + 4 * (32 * d + 2 * e + 4 * h)) =
                    make_float4(acc[d][e] * f, acc[d][e + 1] * f, acc[d][e + 2] * f, acc[d][e + 3] * f);
        if (wave == 0 && h == 0) {
            const i64 rr = (i64)nk * M + r;
            if (out.splits > 1) {
                if (row_ok) {
                    float *ml = out.part + (i64)out.splits * out.rows * c.D + 2 * ((i64)split * out.rows + rr);
                    ml[0] = all;
                    ml[1] = total;
                }
            } else if (out.lse != nullptr && row_ok) {
                out.lse[((i64)n * c.Hq + head) * c.Tq + i] = total == 0.0f ? -INFINITY : all * kLn2 + logf(total);
            }
        }
        // (lane li of every wave has row li's total)
        __syncthreads();
        if (wave == 0 && h == 0) join[0][0][li] = inverse_sum(total, all);
        __syncthreads();
        bool bad = false;
        for (int at = threadIdx.x; at < 32 * (DP / 4); at += S::THREADS) {
            const int row = at / (DP / 4), d = 4 * (at - row * (DP / 4)), rr = r0 + row;
            if (rr >= M || d >= c.D) continue;
            float v[4] = {};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float4 x = *reinterpret_cast<const float4 *>(smem + (w * 32 + row) * S::OUT_ROW + 4 * d);
                v[0] += x.x;
                v[1] += x.y;
                v[2] += x.z;
                v[3] += x.w;
            }
            if (out.splits > 1) {
                float *o = out.part + ((i64)split * out.rows + (i64)nk * M + rr) * c.D + d;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < c.D) o[e] = v[e];
            } else {
                const float inv = join[0][0][row];
                const int ir = rr / c.G;
                T *o = (T *)out.O + ((i64)n * c.Tq + ir) * c.ldo + (i64)(kv * c.G + rr - ir * c.G) * c.D + d;
                bad = bad || not_finite(inv);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] *= inv;
                    bad = bad || not_finite(v[e]);
                    if (d + e < c.D) store_elem(o + e, v[e]);
                }
            }
        }
        wait_loads();                                    // the stores above come before those below
        if (out.splits == 1 && __syncthreads_or(bad))
            for (int k = wave; k < 32 && r0 + k < M; k += NW) {
                const int ik = (r0 + k) / c.G;
                forward_row<T>(c, n, kv * c.G + (r0 + k) - ik * c.G, ik, (T *)out.O, out.lse);
            }
    }
}

// A workgroup joins a row's sums over the splits: its waves take every fourth, eight loads in flight (a loop of single loads over
// 32 splits took 30 us), and are added in wave order.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(Call c, ForwardOut out)
{
    constexpr int NW = 4, PER = kTileD / kWave, AHEAD = 8;
    __shared__ float part[NW][kTileD];
    const i64 rr = blockIdx.x;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int M = c.Tq * c.G, nk = (int)(rr / M), r = (int)(rr - (i64)nk * M);
    const int n = nk / c.Hk, kv = nk - n * c.Hk, i = r / c.G, head = kv * c.G + r - i * c.G;
    const float *ml = out.part + (i64)out.splits * out.rows * c.D + 2 * rr;
    const i64 step = 2 * out.rows;
    float all = -INFINITY;
    for (int s = lane; s < out.splits; s += kWave) all = fmaxf(all, ml[s * step]);
    all = wave_max(all);
    const float base = all == -INFINITY ? 0.0f : all;
    float total = 0.0f;
    for (int s = lane; s < out.splits; s += kWave) total += __builtin_amdgcn_exp2f(ml[s * step] - base) * ml[s * step + 1];
    total = wave_sum(total);
    float v[PER] = {};
    for (int s0 = wave; s0 < out.splits; s0 += NW * AHEAD) {
        float f[AHEAD], x[AHEAD][PER];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int s = s0 + NW * a;
            const bool ok = s < out.splits;
            f[a] = ok ? ml[s * step] : -INFINITY;
            const float *p = out.part + ((i64)(ok ? s : s0) * out.rows + rr) * c.D;
#pragma unroll
            for (int k = 0; k < PER; ++k) x[a][k] = lane + kWave * k < c.D ? p[lane + kWave * k] : 0.0f;
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const float g = __builtin_amdgcn_exp2f(f[a] - base);
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (s0 + NW * a < out.splits) v[k] += g * x[a][k];
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) part[wave][lane + kWave * k] = v[k];
    __syncthreads();
    if (wave != 0) return;
    const float inv = inverse_sum(total, all);
    T *o = (T *)out.O + ((i64)n * c.Tq + i) * c.ldo + (i64)head * c.D;
    bool bad = not_finite(inv) || not_finite(total);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int d = lane + kWave * k;
        v[k] = (((part[0][d] + part[1][d]) + part[2][d]) + part[3][d]) * inv;
        bad = bad || not_finite(v[k]);
    }
    if (__any(bad)) {
        forward_row<T>(c, n, head, i, (T *)out.O, out.lse);
        return;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (lane + kWave * k < c.D) store_elem(o + lane + kWave * k, v[k]);
    if (out.lse != nullptr && lane == 0)
        out.lse[((i64)n * c.Hq + head) * c.Tq + i] = total == 0.0f ? -INFINITY : all * kLn2 + logf(total);
}

template <typename T, int DP, bool VEC, int MOD, bool SMALL>
void launch(const Call &c, const ForwardOut &out, bool vec_out, hipStream_t stream)
{
    typedef Shape<T, DP, SMALL> S;
    const int tiles = (int)ceil_div((i64)c.Tq * c.G, S::BR);
    const unsigned grid = (unsigned)((i64)c.N * c.Hk * tiles * (SMALL ? out.splits : 1));
    forward_kernel<T, DP, VEC, MOD, SMALL><<<grid, S::THREADS, 0, stream>>>(c, out, tiles, vec_out);
}

template <typename T, int DP>
void by_kind(const Call &c, const ForwardOut &out, bool small, hipStream_t stream)
{
    constexpr int N = 16 / sizeof(T);
    const bool vec = c.D % N == 0 && c.ldq % N == 0 && c.ldk % N == 0 && c.ldv % N == 0 && aligned(c.Q, 16) && aligned(c.K, 16) &&
                     aligned(c.V, 16);
    const bool vec_out = c.D % N == 0 && c.ldo % N == 0 && aligned(out.O, 16);
    const int mod = c.scale <= 0.0f ? kBoth : (c.cap > 0.0f ? kCap : kPlain) | (c.slopes != nullptr ? kSlope : kPlain);
    const auto go = [&](auto v, auto m) __attribute__((always_inline)) {
        if (small) launch<T, DP, decltype(v)::value, decltype(m)::value, true>(c, out, vec_out, stream);
        else launch<T, DP, decltype(v)::value, decltype(m)::value, false>(c, out, vec_out, stream);
    };
    if (!vec) go(std::false_type{}, std::integral_constant<int, kBoth>{});
    else if (mod == kPlain) go(std::true_type{}, std::integral_constant<int, kPlain>{});
    else if (mod == kCap) go(std::true_type{}, std::integral_constant<int, kCap>{});
    else if (mod == kSlope) go(std::true_type{}, std::integral_constant<int, kSlope>{});
    else go(std::true_type{}, std::integral_constant<int, kBoth>{});
}

template <typename T>
dp_status tiles_of(const Call &c, const ForwardOut &out, bool small, hipStream_t stream)
{
    if (c.D <= 32) by_kind<T, 32>(c, out, small, stream);
    else if (c.D <= 64) by_kind<T, 64>(c, out, small, stream);
    else if (c.D <= 96) by_kind<T, 96>(c, out, small, stream);
    else by_kind<T, 128>(c, out, small, stream);
    if (out.splits > 1) join_kernel<T><<<(unsigned)out.rows, 256, 0, stream>>>(c, out);
    return launch_status();
}

}  // namespace
}  // namespace attn
}  // namespace dpg
