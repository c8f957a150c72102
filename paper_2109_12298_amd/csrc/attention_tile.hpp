// What the attention tile kernels share: operand tiles in LDS, matrix products
// over them, scores, and which tiles of keys a block of rows meets.
//
// Rows.  The query heads that share a key head run over the same keys, so a
// key head's rows are its (query, head) pairs, r = i * G + g: one product
// serves prompts, shared heads and single tokens alike, and a key head's
// gradients add over its query heads inside a workgroup.
//
// Operands.  A 32 x 32 product of a wave has its two operands' values in pieces
// of 16 bytes: lane l has row l % 32 and the piece l / 32 of a 32-byte k-step
// (bf16: one v_mfma_f32_32x32x16; fp32: four v_mfma_f32_32x32x2, whose two k are
// the two halves' same element: the order of a sum's terms is free as long as
// both operands have the same).  Register r of the result is row
// 8 * (r / 4) + 4 * (l / 32) + r % 4, column l % 32.  With scores formed as
// keys x rows (or rows x keys), a lane has 16 scores of one column, and they
// are, as they lie, the second operand of the product that sums over them:
// bf16 takes registers 8 c .. 8 c + 7 as k = 16 c + {4 h .. 4 h + 3, 8 + 4 h ..
// 8 + 4 h + 3} (h = l / 32), fp32 register r alone.  The first operand is then
// the other tile read by columns: transposing LDS reads in bf16 (four rows
// each), plain ones in fp32.
//
// Tiles.  Rows of DP values (D rounded up to 32; what is behind D repeats the
// row's first piece and meets zeros in the other operand), 16-byte piece q of
// row r at place q ^ swz(r): 16 rows' same pieces lie in 16 different places of
// the 256-byte bank window, and 4 rows' same 64 bytes in 4.
#pragma once

#include "attention_rows.hpp"
#include "bf16_stage.hpp"

namespace dpg {
namespace attn {

using bf16s::bf16x8_t;
using bf16s::f32x16_t;
using bf16s::i16x4_t;
using bf16s::i16x8_t;
using bf16s::lds_addr;
using bf16s::lds_i16x4_t;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// a pointer that is the same in all lanes, in scalar registers
template <typename P>
__device__ __forceinline__ P *uniform(P *p)
{
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<P *>((uint64_t)hi << 32 | lo);
}

// lane l's 16 (4) bytes at base + off go to LDS byte lds + 16 l (4 l); see bf16s::dma16
__device__ __forceinline__ void dma16_off(const void *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(uniform(base)),
                 "s"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory", "m0");
}
__device__ __forceinline__ void dma4_off(const void *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(uniform(base)),
                 "s"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory", "m0");
}

__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// All lanes of the wave go on from here together.  The matrix instructions and LDS reads are not marked as ones that a wave runs
// as a whole: a lane-dependent branch right before a loop of them was once drawn into the loop, whose trips then ran with some
// lanes switched off.
__device__ __forceinline__ void wave_together() { __builtin_amdgcn_wave_barrier(); }

// the value of lane ^ 32
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, kWave); }

template <typename T, int DP_>
struct Tile {
    static constexpr int DP = DP_, RB = DP * (int)sizeof(T), PIECES = RB / 16, KS = RB / 32, DB = DP / 32;
    static constexpr int N = 16 / (int)sizeof(T);                // values in a piece
    static constexpr bool BF16 = sizeof(T) == 2;

    static __device__ __forceinline__ int swz(int r)
    {
        if constexpr (BF16) {
            if constexpr (RB % 256 == 0) return ((r & 3) << 2) | ((r >> 2) & 3);
            else if constexpr (RB % 256 == 128) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
            else return (r >> 2) & 3;
        } else {
            // rows four apart, which the two halves of a wave read together, in different halves of the window
            if constexpr (RB % 256 == 0) return (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1);
            else return (r >> 1) & 7;
        }
    }

    // operand of the rows r0 .. r0 + 31 at k-step ks
    static __device__ __forceinline__ u32x4_t rows(const char *L, int r0, int ks, int lane)
    {
        const int r = r0 + (lane & 31);
        return *reinterpret_cast<const u32x4_t *>(L + r * RB + 16 * ((2 * ks + (lane >> 5)) ^ swz(r)));
    }
    // sum of the products of two pieces' values
    static __device__ __forceinline__ float dot(const u32x4_t &a, const u32x4_t &b)
    {
        float v = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF16) {
                v = __builtin_fmaf(__uint_as_float(a[e] << 16), __uint_as_float(b[e] << 16), v);
                v = __builtin_fmaf(__uint_as_float(a[e] & 0xffff0000u), __uint_as_float(b[e] & 0xffff0000u), v);
            } else {
                v = __builtin_fmaf(__uint_as_float(a[e]), __uint_as_float(b[e]), v);
            }
        }
        return v;
    }
    static __device__ __forceinline__ void mma(const u32x4_t &a, const u32x4_t &b, f32x16_t &acc)
    {
        if constexpr (BF16) {
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc,
                                                          0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
        }
    }
    // The products below are given by what their steps read, take and add to.  LDS reads run ahead of the matrix instructions that
    // take them, kept there by scheduling barriers that neither may cross: left to itself the compiler keeps registers low by a
    // read right before each, whose latency the wave then waits for (two prompts of 4096, 32 and 8 heads of 128: 325 us; 294 with them ahead).
    static __device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x6); }

    // acc(i) += read(i, ks) x operand(i, ks) over all k-steps, for COUNT products side by side
    template <int COUNT, int STEPS_AHEAD = 2, typename Read, typename Operand, typename Acc>
    static __device__ __forceinline__ void products(Read &&read, Operand &&operand, Acc &&acc)
    {
        constexpr int AHEAD = KS < STEPS_AHEAD ? KS : STEPS_AHEAD, BUFS = AHEAD + 1;
        u32x4_t f[BUFS][COUNT];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) f[k][i] = read(i, k);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + AHEAD < KS)
#pragma unroll
                for (int i = 0; i < COUNT; ++i) f[(ks + AHEAD) % BUFS][i] = read(i, ks + AHEAD);
            keep_order();
#pragma unroll
            for (int i = 0; i < COUNT; ++i) mma(f[ks % BUFS][i], operand(i, ks), acc(i));
            keep_order();
        }
    }

    // acc(i)[block of 32 values][.] += sum over 32 rows r of tile(i)[r][value] * w(i)[r], for COUNT blocks of rows one after
    // another; tile(i): where the block starts (a multiple of 32 rows of a tile).
    // bf16 products take w rounded to bf16; where bit i of SPLIT is set, as the sum of two bf16 values, whose second product reads
    // nothing anew.  also(step, d, operand): further products of what was read (bf16).
    struct Nothing {
        __device__ __forceinline__ void operator()(int, int, const bf16x8_t &) const {}
    };
    template <int COUNT, unsigned SPLIT = 0, typename At, typename W, typename Acc, typename Also = Nothing>
    static __device__ __forceinline__ void columns(At &&tile, W &&w, Acc &&acc, int lane, Also &&also = Also())
    {
        const int h = lane >> 5;
        if constexpr (BF16) {
            const int s = lane & 15, g = (lane >> 4) & 1;
            const auto load = [&](int step, bf16x8_t (&a)[DB]) {
                const char *L = tile(step >> 1);
                const int t = 16 * (step & 1) + 4 * h + (s >> 2);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const int q = 4 * d + 2 * g + ((s & 3) >> 1), in = 8 * (s & 1);
                    const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(L + t * RB + 16 * (q ^ swz(t)) + in));
                    const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_i16x4_t *)(L + (t + 8) * RB + 16 * (q ^ swz(t + 8)) + in));
                    a[d] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            };
            bf16x8_t a[2][DB];
            load(0, a[0]);
#pragma unroll
            for (int step = 0; step < 2 * COUNT; ++step) {
                if (step + 1 < 2 * COUNT) load(step + 1, a[(step + 1) & 1]);
                const bool split = (SPLIT >> (step >> 1) & 1) != 0;
                bf16x8_t b, rest;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = w(step >> 1)[8 * (step & 1) + e];
                    b[e] = (__bf16)x;
                    if (split) rest[e] = (__bf16)(x - (float)b[e]);
                }
                keep_order();
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    acc(step >> 1)[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[step & 1][d], b, acc(step >> 1)[d], 0, 0, 0);
                    if (split)
                        acc(step >> 1)[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[step & 1][d], rest, acc(step >> 1)[d], 0, 0, 0);
                    also(step, d, a[step & 1][d]);
                }
                keep_order();
            }
        } else {
            const auto load = [&](int step, float (&a)[DB]) {
                const char *L = tile(step >> 4);
                const int r = step & 15, t = 8 * (r >> 2) + 4 * h + (r & 3);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const int v = 32 * d + (lane & 31);
                    a[d] = *reinterpret_cast<const float *>(L + t * RB + 16 * ((v >> 2) ^ swz(t)) + 4 * (v & 3));
                }
            };
            float a[3][DB];
            load(0, a[0]);
            load(1, a[1]);
#pragma unroll
            for (int step = 0; step < 16 * COUNT; ++step) {
                if (step + 2 < 16 * COUNT) load(step + 2, a[(step + 2) % 3]);
                keep_order();
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    acc(step >> 4)[d] =
                        __builtin_amdgcn_mfma_f32_32x32x2f32(a[step % 3][d], w(step >> 4)[step & 15], acc(step >> 4)[d], 0, 0, 0);
                keep_order();
            }
        }
    }

    // A row's operands for all k-steps, from memory; zeros behind D and where !ok (the row is one that may be read all the same).
    // No branches: the values are lanes' own, and what follows has to be run by all lanes together.
    static __device__ __forceinline__ void load_row(const T *p, int D, bool ok, bool vec, int lane, u32x4_t (&f)[KS])
    {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = (2 * ks + (lane >> 5)) * N;
            u32x4_t v = vec ? *reinterpret_cast<const u32x4_t *>(p + (d < D ? d : 0)) : piece(p, d, D);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ok && d < D ? v[e] : 0;
            f[ks] = v;
        }
    }
    // values d .. of a row of any alignment, zeros from D on (a value behind the end is loaded from the row's first place)
    static __device__ __forceinline__ u32x4_t piece(const T *p, int d, int D)
    {
        u32x4_t v = {0, 0, 0, 0};
        if constexpr (BF16) {
            uint32_t x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = p[d + e < D ? d + e : 0];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e >> 1] |= (d + e < D ? x[e] : 0) << (16 * (e & 1));
        } else {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = p[d + e < D ? d + e : 0];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = d + e < D ? __float_as_uint(x[e]) : 0;
        }
        return v;
    }
};

// Brings R rows of a tile to LDS with NW waves: places are formed once, and again only for a tile that ends early.
template <typename TL, typename T, int R, int NW, bool VEC>
struct Stager {
    static constexpr int LOADS = R * TL::RB / 1024 / NW;
    static_assert(LOADS * NW * 1024 == R * TL::RB, "stage split");
    // 16 rows on, a place is the same but for the rows: PERIOD places, the others by the base
    static constexpr bool WHOLE = 64 * NW % TL::PIECES == 0;
    static constexpr int STEP = WHOLE ? 64 * NW / TL::PIECES : 1;        // rows from one load to the next
    static constexpr int EVERY = !WHOLE ? LOADS : STEP % 16 == 0 ? 1 : 16 % STEP == 0 ? 16 / STEP : LOADS;
    static constexpr int PERIOD = EVERY < LOADS ? EVERY : LOADS;

    uint32_t ld_bytes, off[VEC ? PERIOD : 1];
    int D, wave, lane;

    __device__ __forceinline__ Stager(i64 ld, int D_, int wave_, int lane_)
        : ld_bytes((uint32_t)(ld * sizeof(T))), D(D_), wave(wave_), lane(lane_)
    {
        if constexpr (VEC)
#pragma unroll
            for (int k = 0; k < PERIOD; ++k) {
                int row, q;
                place(k, row, q);
                off[k] = (uint32_t)row * ld_bytes + byte(q);
            }
    }
    __device__ __forceinline__ void place(int k, int &row, int &piece) const
    {
        const int at = 64 * (wave + NW * k) + lane;
        row = at / TL::PIECES;
        piece = (at - row * TL::PIECES) ^ TL::swz(row);
    }
    __device__ __forceinline__ uint32_t byte(int q) const { return 16u * (uint32_t)(q * TL::N < D ? q : 0); }
    // Rows from `left` on read the one before it, those before `skip` that one: their weights are zeros, and what lies in their own
    // places (padding may hold anything) meets no product.
    __device__ __forceinline__ void issue(const T *base, int left, uint32_t lds, char *generic, int skip = 0) const
    {
        if constexpr (VEC) {
            if (left >= R && skip <= 0) {
#pragma unroll
                for (int k = 0; k < LOADS; ++k)
                    dma16_off(reinterpret_cast<const char *>(base) + (i64)(k / PERIOD * PERIOD * STEP) * ld_bytes, off[k % PERIOD],
                              lds + 1024u * (uint32_t)(wave + NW * k));
                return;
            }
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            int row, q;
            place(k, row, q);
            const int in = row < skip ? skip : row, r = in < left ? in : left - 1;
            if constexpr (VEC) {
                dma16_off(base, (uint32_t)r * ld_bytes + byte(q), lds + 1024u * (uint32_t)(wave + NW * k));
            } else {
                const T *p = reinterpret_cast<const T *>(reinterpret_cast<const char *>(base) + (i64)r * ld_bytes);
                *reinterpret_cast<u32x4_t *>(generic + 1024 * (wave + NW * k) + 16 * lane) = TL::piece(p, q * TL::N, D);
            }
        }
    }
};

// ---------------------------------------------------------------------------
// scores in units of ln 2
// ---------------------------------------------------------------------------
// What a score has besides its scale (> 0): kBoth looks at run time, and takes any scale
enum { kPlain = 0, kCap = 1, kSlope = 2, kBoth = 3 };

// tanh y = y P(y^2) up to |y| = 3/4 (least-maximum fits: five terms within 6e-7
// of it for scores of bf16 inputs, whose rounding is 2^-9 of a score, seven within
// 1.5e-9 for fp32 ones), from there 1 - 2 / (1 + exp 2|y|), whose subtrahend is at
// most 0.37 and off by some 2^-23 of it.  With r = 1 / (1 + exp 2|y|), 1 - tanh^2 is
// 4 r (1 - r), which keeps its digits where tanh is all but 1.  Where no score of a bf16 wave's block
// goes past 3/4, which a cap is chosen for, the polynomial alone is taken, with
// the scales in its coefficients: five instructions a score, of which the last
// forms the exponent.  No branches by lane: see wave_together.
constexpr float kNear = 0.75f;
constexpr float kTanh[5] = {0.999999435f, -0.333282516f, 0.132589834f, -0.0500563036f, 0.0129296314f};

constexpr float kTanh7[7] = {0.999999999f, -0.33333307f, 0.133325791f, -0.0538856315f, 0.0214308735f, -0.00762702948f, 0.00172035412f};

template <typename T>
__device__ __forceinline__ float tanh_for(float y, float &bend)
{
    constexpr int TERMS = sizeof(T) == 2 ? 5 : 7;
    const float a = __builtin_fabsf(y), u = y * y;
    float p = sizeof(T) == 2 ? kTanh[4] : kTanh7[6];
#pragma unroll
    for (int k = TERMS - 2; k >= 0; --k) p = __builtin_fmaf(u, p, sizeof(T) == 2 ? kTanh[k] : kTanh7[k]);
    const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(2.0f * kLog2e * a)), far = 1.0f - 2.0f * r;
    bend = 4.0f * r * (1.0f - r);
    return a < kNear ? y * p : __builtin_copysignf(far, y);
}

template <typename T, int MOD>
struct Scores {
    float scale2;            // scale * log2 e
    float y_scale, cap2;     // scale / cap, cap * log2 e; cap2 = 0: no cap
    float inv_cap2;          // 1 / cap2
    float c[5];              // the polynomial's, of the raw score
    float near_to;           // |y| up to which it holds; -1 where its coefficients might overflow

    __device__ __forceinline__ explicit Scores(const Call &a)
    {
        scale2 = a.scale * kLog2e;
        cap2 = a.cap * kLog2e;
        y_scale = a.cap > 0.0f ? a.scale / a.cap : 0.0f;
        inv_cap2 = a.cap > 0.0f ? 1.0f / cap2 : 0.0f;
        float f = cap2 * y_scale;
#pragma unroll
        for (int k = 0; k < 5; ++k, f *= y_scale * y_scale) c[k] = f * kTanh[k];
        near_to = __builtin_fabsf(y_scale) <= 1024.0f && __builtin_fabsf(scale2) <= 0x1p40f ? kNear : -1.0f;
    }
    // whether the polynomial may be taken for all raw scores of the wave's block
    __device__ __forceinline__ bool near(const f32x16_t &x) const
    {
        if constexpr (MOD != kCap || sizeof(T) != 2) return false;
        float m = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, __builtin_fabsf(x[e]));
        return !__any(!(m * __builtin_fabsf(y_scale) <= near_to));
    }
    __device__ __forceinline__ float poly(float x) const
    {
        const float u = x * x;
        return __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, c[4], c[3]), c[2]), c[1]), c[0]);
    }
    // a raw score less `base`; bend: the capped score's derivative by the uncapped one
    template <bool NEAR>
    __device__ __forceinline__ float of(float x, float base, float slope2, float far, float &bend) const
    {
        bend = 1.0f;
        if constexpr (MOD == kPlain) {
            return __builtin_fmaf(x, scale2, -base);
        } else if constexpr (MOD == kSlope) {
            return __builtin_fmaf(-slope2, far, __builtin_fmaf(x, scale2, -base));
        } else if constexpr (MOD == kCap) {
            if constexpr (NEAR) {
                const float p = poly(x), t = x * p * inv_cap2;
                bend = __builtin_fmaf(-t, t, 1.0f);
                return __builtin_fmaf(x, p, -base);
            } else {
                const float t = tanh_for<T>(y_scale * x, bend);
                return __builtin_fmaf(cap2, t, -base);
            }
        } else {
            float v = scale2 * x;
            if (cap2 != 0.0f) {
                v = cap2 * tanh_for<T>(y_scale * x, bend);
            }
            return v - slope2 * far - base;
        }
    }
};

// ---------------------------------------------------------------------------
// which tiles two blocks meet in
// ---------------------------------------------------------------------------
// A block of rows: the positions of its valid rows and their documents
struct RowSpan {
    int pmin, pmax;          // pmax < pmin: none is valid
    bool all;                // every row of the block is valid
    int dmin, dmax;          // their documents' range (with docs; -1 .. : one may be negative)
};

// r0 .. r0 + count - 1 of M rows
__device__ __forceinline__ RowSpan span_of(const Sample &s, int G, int M, int r0, int count)
{
    RowSpan b;
    const int last = r0 + count < M ? r0 + count : M;
    const int p0 = s.first + r0 / G, p1 = s.first + (last - 1) / G;
    b.pmin = p0 > 0 ? p0 : 0;
    b.pmax = p1 < s.L ? p1 : s.L - 1;
    if (last <= r0) b.pmax = b.pmin - 1;
    b.all = r0 + count <= M && p0 >= 0 && p1 < s.L;
    b.dmin = b.dmax = 0;
    return b;
}

// kDocs: partial, and documents have to be compared
enum { kSkip = 0, kPartial = 1, kFull = 2, kDocs = 3 };

// keys [k0, k1) against the span; kd0, kd1: the documents' range of those below L
__device__ __forceinline__ int meet(const Sample &s, const RowSpan &b, int k0, int k1, int kd0, int kd1)
{
    if (b.pmax < b.pmin || k0 >= s.end_for(b.pmax)) return kSkip;
    bool full = b.all && k1 <= s.L && (!s.causal || k1 - 1 <= b.pmin || k1 <= s.prefix);
    if (s.docs != nullptr) {
        if (kd1 < 0 || b.dmax < 0 || kd1 < b.dmin || kd0 > b.dmax) return kSkip;
        if (kd0 != kd1 || b.dmin != b.dmax) return kDocs;
    }
    return full ? kFull : kPartial;
}

// range of docs[j0 .. j1)
__device__ __forceinline__ void docs_range(const int32_t *docs, int j0, int j1, int &lo, int &hi)
{
    lo = 0x7fffffff;
    hi = -0x7fffffff - 1;
    int j = j0;
    for (; j + 8 <= j1; j += 8) {
        int v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = docs[j + k];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            lo = v[k] < lo ? v[k] : lo;
            hi = v[k] > hi ? v[k] : hi;
        }
    }
    for (; j < j1; ++j) {
        lo = docs[j] < lo ? docs[j] : lo;
        hi = docs[j] > hi ? docs[j] : hi;
    }
}

__device__ __forceinline__ bool not_finite(float v) { return !(__builtin_fabsf(v) < INFINITY); }

// 1 / sum of a row's weights, taken from the maximum `top`: 0 for a row that sees nothing, NaN for one that has to be formed again.
// A weight's exponent is a fused product less the rounded one of the maximum, so that the largest weight is 2^(rounding of top), not
// 1: from scores of 2^29 on (in units of ln 2) the roundings reach 2^5, from 2^31 on all weights may vanish, or overflow.
__device__ __forceinline__ float inverse_sum(float sum, float top)
{
    if (sum == 0.0f && top == -INFINITY) return 0.0f;
    return sum < 0x1p-32f ? NAN : 1.0f / sum;
}

}  // namespace attn
}  // namespace dpg
