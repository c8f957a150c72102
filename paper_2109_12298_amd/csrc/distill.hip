// Distillation from a teacher's top logits, and cross entropy, with the gradient.
//
// With q_t = softmax(z / t) and P the teacher's softmax over its K logits,
//   loss = w (a tau^2 sum P (log P - log q_tau) + (1 - a) (-log q_1[label]))
//   dz   = w (a tau (q_tau - P) + (1 - a) (q_1 - onehot)).
// Bound by its bytes: the logits are read once and the gradient written once.
// One workgroup takes a position.  Rows that fit its registers stay there
// between the three steps (maximum; sums of exponentials; gradient), so that
// they are read once; longer rows are read again, by the same threads.  The
// gradient leaves for the whole row as if no class had a target; after a
// barrier (which waits for the stores) the at most K + 1 target classes are
// written anew, each formed in fp32 from its own logit and rounded once.  Those
// logits are read before the first store, so dZ may be Z.
//
// 1001 rows of 32001, bf16, labels mixed in: 39 us (26 at a copy's rate: four
// workgroups a CU at most, each waiting for its own row).  8192 rows of 100000: 790
// us, 4.2 TB/s; a row fills a CU's registers, so that its loads, exponentials and
// stores do not overlap with another row's.  256 rows of 10000, fp32: 8 us.
//
// Rows start at any element: up to 16 / sizeof(T) - 1 elements before the first
// 16-byte piece and behind the last one are single loads and stores.
#include "common.hpp"

#include <type_traits>

namespace dpg {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxK = 1024;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint16_t bf16_bits(float x)
{
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = bf16_bits(v); }

// element e of a 16-byte piece
template <typename T>
__device__ __forceinline__ float elem(u32x4_t v, int e)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
    else return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
}

// piece of f(0) .. f(N - 1)
template <typename T, typename F>
__device__ __forceinline__ u32x4_t piece(F &&f)
{
    u32x4_t v;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(f(e));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (uint32_t)bf16_bits(f(2 * e)) | ((uint32_t)bf16_bits(f(2 * e + 1)) << 16);
    }
    return v;
}

struct Args {
    i64 V;
    const int64_t *ids;
    const float *logits;
    int K;
    const int64_t *labels;
    float alpha, tau;
    const float *weight;
    float *loss;
    int32_t *status;
};

// Maxima (a NaN is passed over here and turns the sums to NaN) and sums over the
// workgroup, several at once, as each costs a barrier; every thread gets the results.
__device__ __forceinline__ float wave_max(float v)
{
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, kWave));
    return v;
}
// `red` (N values a wave) is not used again before a barrier
template <int THREADS, int N>
__device__ __forceinline__ void block_max(float (&v)[N], float (*red)[16])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_max(v[i]);
    if constexpr (THREADS > kWave) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i][threadIdx.x >> 6] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = red[i][0];
#pragma unroll
            for (int w = 1; w < THREADS / kWave; ++w) v[i] = fmaxf(v[i], red[i][w]);
        }
    }
}
template <int THREADS, int N>
__device__ __forceinline__ void block_add(float (&v)[N], float (*red)[16])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (THREADS > kWave) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i][threadIdx.x >> 6] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < THREADS / kWave; ++w) v[i] += red[i][w];
        }
    }
}

// NV pieces of a row per thread are held; RESIDENT: they are the whole row.
// HARD: labels have a share of the loss (a position may lack its own).
template <typename T, int THREADS, int NV, bool RESIDENT, bool HARD>
__global__ __launch_bounds__(THREADS) void distill_kernel(const T *Z, i64 M, Args a, T *dZ)
{
    constexpr int N = 16 / sizeof(T);
    __shared__ float red[6][16];                           // two maxima, three sums, the loss
    __shared__ float target[kMaxK];                        // P_k
    __shared__ int32_t target_id[kMaxK];                   // -1: unused
    const i64 V = a.V;
    const int tid = threadIdx.x;
    const i64 m = (i64)blockIdx.y * gridDim.x + blockIdx.x;
    if (m >= M) return;
    const T *z = Z + m * V;
    T *dz = dZ != nullptr ? dZ + m * V : nullptr;
    const float w = a.weight != nullptr ? a.weight[m] : 1.0f;

    const int head = (int)(((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / sizeof(T));
    const int first = head < V ? head : (int)V;
    const int pieces = (int)((V - first) / N);
    const int rest = first + pieces * N;                   // first element behind the pieces
    const bool vec = dz != nullptr && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
    // the single element of this thread, if any
    const int single = tid < first ? tid : tid < first + (int)V - rest ? rest + tid - first : -1;

    const auto leave_out = [&]() {
        if (dz != nullptr) {
            for (int p = tid; p < pieces; p += THREADS)
                if (vec) *reinterpret_cast<u32x4_t *>(dz + first + (i64)p * N) = u32x4_t{0, 0, 0, 0};
                else
                    for (int e = 0; e < N; ++e) put(dz + first + (i64)p * N + e, 0.0f);
            if (single >= 0) put(dz + single, 0.0f);
        }
        if (tid == 0) a.loss[m] = 0.0f;
    };
    // All loads leave before the first is waited for: the row's, the label's, the teacher's and, behind its ids, the target classes'
    // own logits (which are read before any store).
    u32x4_t v[NV];
    const auto load = [&](int base) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = base + i * THREADS + tid;
            if (p < pieces) {
                const u32x4_t *at = reinterpret_cast<const u32x4_t *>(z + first + (i64)p * N);
                v[i] = RESIDENT ? __builtin_nontemporal_load(at) : *at;
            }
        }
    };
    int64_t wanted = -1;
    if (HARD || a.labels != nullptr) wanted = a.labels[m];
    constexpr int PER = (kMaxK + THREADS - 1) / THREADS;
    int64_t id_of[PER];
    float logit_of[PER], mine[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = tid + i * THREADS;
        id_of[i] = k < a.K ? a.ids[m * a.K + k] : -1;
        logit_of[i] = k < a.K ? a.logits[m * a.K + k] : -INFINITY;
    }
    if constexpr (RESIDENT) load(0);
    float one = -INFINITY;
    if (single >= 0) one = load_elem<T>(z, single);
    const int label = HARD && wanted >= 0 && wanted < V ? (int)wanted : -1;
    const bool hard = HARD && label >= 0 && a.alpha < 1.0f;
    const float z_label = hard ? load_elem<T>(z, label) : 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine[i] = id_of[i] >= 0 && id_of[i] < V ? load_elem<T>(z, id_of[i]) : 0.0f;
    if (w == 0.0f) {
        leave_out();
        return;
    }
    const float inv_tau = 1.0f / a.tau, c_tau = kLog2e * inv_tau;
    float tmax = -INFINITY;
    bool bad_id = tid == 0 && wanted >= V;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = tid + i * THREADS;
        if (k >= a.K) break;
        const bool ok = id_of[i] >= 0 && id_of[i] < V;
        bad_id = bad_id || id_of[i] >= V;
        target_id[k] = ok ? (int32_t)id_of[i] : -1;
        target[k] = ok ? logit_of[i] : -INFINITY;
        tmax = fmaxf(tmax, target[k]);
    }
    if (bad_id) raise_flag(a.status, DP_FLAG_BAD_INDEX);
    // the teacher's and the row's maxima, then the sums of exponentials
    float zmax = one, s_tau = 0.0f, s_1 = 0.0f;
    // exp((x - top) / t) as a power of 2.  In general the difference comes first, which is exact where it is small.  A row in registers
    // whose top / t is below 2^24 takes one fused product instead, x / t less the rounded top / t, whose rounding is one factor of all
    // of the row's exponentials, within 2^0.5, and so none of a softmax (8192 rows of 100000, bf16: 787 us, 823 by differences).  From
    // 2^31 on that factor would vanish or overflow, and sums taken from several maxima would each have their own.
    const bool same = a.tau == 1.0f;                       // one exponential serves both
    const auto power = [&](auto fused, float x, float base, float c) {
        return decltype(fused)::value ? __builtin_fmaf(x, c, -(base * c)) : (x - base) * c;
    };
    const auto add = [&](auto fused, float x, float base) {
        const float e = __builtin_amdgcn_exp2f(power(fused, x, base, c_tau));
        s_tau += e;
        if constexpr (HARD) s_1 += same ? e : __builtin_amdgcn_exp2f(power(fused, x, base, kLog2e));
    };
    const auto by = [&](bool fused, auto &&f) {
        if (fused) f(std::true_type{});
        else f(std::false_type{});
    };
    float top = -INFINITY;                                 // !RESIDENT: the maximum that this thread's sums are taken from
    if constexpr (RESIDENT) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * THREADS + tid < pieces)
#pragma unroll
                for (int e = 0; e < N; ++e) zmax = fmaxf(zmax, elem<T>(v[i], e));
    } else {
        for (int base = 0; base < pieces; base += NV * THREADS) {
            load(base);
            float t = top;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (base + i * THREADS + tid < pieces)
#pragma unroll
                    for (int e = 0; e < N; ++e) t = fmaxf(t, elem<T>(v[i], e));
            if (t > top) {
                s_tau *= __builtin_amdgcn_exp2f((top - t) * c_tau);
                if constexpr (HARD) s_1 *= __builtin_amdgcn_exp2f((top - t) * kLog2e);
                top = t;
            }
            const float base_t = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (base + i * THREADS + tid < pieces)
#pragma unroll
                    for (int e = 0; e < N; ++e) add(std::false_type{}, elem<T>(v[i], e), base_t);
        }
        zmax = fmaxf(zmax, top);
    }
    float maxima[2] = {tmax, zmax};
    block_max<THREADS>(maxima, red);
    const float tbase = maxima[0] == -INFINITY ? 0.0f : maxima[0], zbase = maxima[1] == -INFINITY ? 0.0f : maxima[1];
    float tsum = 0.0f;
    for (int k = tid; k < a.K; k += THREADS)
        if (target_id[k] >= 0) tsum += expf((target[k] - tbase) * inv_tau);
    if (!RESIDENT && top != -INFINITY) {
        s_tau *= __builtin_amdgcn_exp2f((top - zbase) * c_tau);
        if constexpr (HARD) s_1 *= __builtin_amdgcn_exp2f((top - zbase) * kLog2e);
    }
    const bool is_fused = RESIDENT && __builtin_fabsf(zbase) * fmaxf(c_tau, kLog2e) < 0x1p24f;
    by(is_fused, [&](auto fused) {
        if (single >= 0) add(fused, one, zbase);
        if constexpr (RESIDENT)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * THREADS + tid < pieces)
#pragma unroll
                    for (int e = 0; e < N; ++e) add(fused, elem<T>(v[i], e), zbase);
    });
    float sums[HARD ? 3 : 2] = {tsum, s_tau};
    if constexpr (HARD) sums[2] = s_1;
    block_add<THREADS>(sums, red + 2);
    tsum = sums[0];
    s_tau = sums[1];
    if constexpr (HARD) s_1 = sums[2];

    const bool soft = a.alpha > 0.0f && tsum != 0.0f;
    const float ltsum = logf(tsum);
    if (!soft && !hard) {                                  // no part of the loss
        leave_out();
        return;
    }

    // P in place of the teacher's logits; the loss, by differences of logits (a fused power's factor log2 e would overflow for the
    // lowest value) and the sums' logarithms less what the fused maximum's own power is off from 0
    const auto log_sum = [&](float sum, float c) {
        return logf(sum) - (is_fused ? kLn2 * power(std::true_type{}, zbase, zbase, c) : 0.0f);
    };
    float part = 0.0f;
    const float lq = log_sum(s_tau, c_tau);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = tid + i * THREADS;
        if (k >= a.K) break;
        float P = 0.0f;
        if (soft && target_id[k] >= 0) {
            const float lp = (target[k] - tbase) * inv_tau - ltsum;
            P = expf(lp);
            if (P != 0.0f) part += P * (lp - ((mine[i] - zbase) * inv_tau - lq));
        }
        target[k] = P;
    }
    float parts[1] = {part};
    if (a.K > kWave) block_add<THREADS>(parts, red + 5);
    else parts[0] = wave_sum(part);                        // the first wave has all of them
    const float g_soft = soft ? a.alpha : 0.0f, g_hard = hard ? 1.0f - a.alpha : 0.0f;
    if (tid == 0) {
        float l = g_soft * a.tau * a.tau * parts[0];
        if (hard) l += g_hard * (log_sum(s_1, kLog2e) - (z_label - zbase));
        a.loss[m] = w * l;
    }
    if (dz == nullptr) return;

    // gradient of a class without a target: w a tau q_tau + w (1 - a) q_1
    const float k_tau = soft ? w * g_soft * a.tau / s_tau : 0.0f, k_1 = hard ? w * g_hard / s_1 : 0.0f;
    const auto grad = [&](auto fused, float x) {
        const float e = __builtin_amdgcn_exp2f(power(fused, x, zbase, c_tau));
        float g = k_tau * e;
        if constexpr (HARD) g += k_1 * (same ? e : __builtin_amdgcn_exp2f(power(fused, x, zbase, kLog2e)));
        return g;
    };
    __syncthreads();
    by(is_fused, [&](auto fused) {
        for (int base = 0; base < (RESIDENT ? 1 : pieces); base += NV * THREADS) {
            if constexpr (!RESIDENT) load(base);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = base + i * THREADS + tid;
                if (p < pieces) {
                    const u32x4_t o = piece<T>([&](int e) { return grad(fused, elem<T>(v[i], e)); });
                    T *at = dz + first + (i64)p * N;
                    if (vec) __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t *>(at));
                    else
#pragma unroll
                        for (int e = 0; e < N; ++e) put(at + e, elem<T>(o, e));
                }
            }
        }
        if (single >= 0) put(dz + single, grad(fused, one));
    });
    __syncthreads();                                       // waits for the stores above

    // target classes: an id that occurs twice is written by its first place, with both
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = tid + i * THREADS;
        if (k >= a.K) break;
        const int32_t id = target_id[k];
        if (id < 0) continue;
        float P = 0.0f;
        bool mine_first = true;
        for (int j = 0; j < a.K; ++j)
            if (target_id[j] == id) {
                P += target[j];
                mine_first = mine_first && j >= k;
            }
        if (!mine_first) continue;
        float g = 0.0f;
        by(is_fused, [&](auto fused) { g = grad(fused, mine[i]) - w * g_soft * a.tau * P; });
        if (id == label) g -= w * g_hard;
        put(dz + id, g);
    }
    if (tid == 0 && hard) {
        bool alone = true;
        for (int j = 0; j < a.K; ++j) alone = alone && target_id[j] != label;
        if (alone) by(is_fused, [&](auto fused) { put(dz + label, grad(fused, z_label) - w * g_hard); });
    }
}

template <typename T, int THREADS, int NV, bool RESIDENT>
void launch(const T *Z, i64 M, const Args &a, T *dZ, hipStream_t stream)
{
    // a dimension of a grid holds fewer than 2^32 threads
    const i64 gx = M < (i64(1) << 20) ? M : i64(1) << 20;
    const dim3 grid((unsigned)gx, (unsigned)ceil_div(M, gx));
    if (a.labels != nullptr && a.alpha < 1.0f)
        distill_kernel<T, THREADS, NV, RESIDENT, true><<<grid, THREADS, 0, stream>>>(Z, M, a, dZ);
    else
        distill_kernel<T, THREADS, NV, RESIDENT, false><<<grid, THREADS, 0, stream>>>(Z, M, a, dZ);
}

template <typename T>
dp_status run(const void *Zp, i64 M, const Args &a, void *dZp, hipStream_t stream)
{
    const T *Z = (const T *)Zp;
    T *dZ = (T *)dZp;
    const i64 pieces = a.V / (16 / (i64)sizeof(T));
    // The fewest threads, and pieces of each, that hold a row: more threads than it has work for cost barriers (4096 rows, bf16: 5000
    // classes 23 us with 256 threads, 55 with 1024), more pieces registers (40000 classes with labels 207 us with 8, 236 with 20;
    // 100000: 445 with 13, 452 with 20), and a second read of the row is what all of it is for (70000: 272 and 335; 160000: 551 and
    // 726; fp32, 80000: 473 and 648).
    if (pieces <= 64 * 4) launch<T, 64, 4, true>(Z, M, a, dZ, stream);
    else if (pieces <= 256 * 4) launch<T, 256, 4, true>(Z, M, a, dZ, stream);
    else if (pieces <= 1024 * 4) launch<T, 1024, 4, true>(Z, M, a, dZ, stream);
    else if (pieces <= 1024 * 8) launch<T, 1024, 8, true>(Z, M, a, dZ, stream);
    else if (pieces <= 1024 * 13) launch<T, 1024, 13, true>(Z, M, a, dZ, stream);
    else if (pieces <= 1024 * 20) launch<T, 1024, 20, true>(Z, M, a, dZ, stream);
    else launch<T, 1024, 8, false>(Z, M, a, dZ, stream);
    return launch_status();
}

}  // namespace
}  // namespace dpg

using namespace dpg;

extern "C" size_t dp_distill_loss_workspace_bytes(int64_t, int64_t, int64_t, dp_dtype) { return 0; }

extern "C" dp_status dp_distill_loss(const void *Z, dp_dtype dt, int64_t M, int64_t V, const int64_t *ids,
                                     const float *logits, int64_t K, const int64_t *labels, float alpha, float tau,
                                     const float *weight, float *loss, void *dZ, int32_t *status, void *, size_t,
                                     hipStream_t stream)
{
    DPG_REQUIRE(dtype_ok(dt), DP_EDTYPE);
    DPG_REQUIRE(M >= 0 && K >= 0 && V >= 1, DP_EINVAL);
    DPG_REQUIRE(alpha >= 0.0f && alpha <= 1.0f && tau >= 0x1p-20f && tau <= 0x1p20f, DP_EINVAL);
    DPG_REQUIRE(M < (i64(1) << 31) && V < (i64(1) << 30) && K <= kMaxK, DP_EUNSUPPORTED);
    if (M == 0) return DP_OK;
    DPG_REQUIRE(Z != nullptr && loss != nullptr && (K == 0 || (ids != nullptr && logits != nullptr)), DP_EINVAL);
    DPG_REQUIRE(aligned(Z, dtype_bytes(dt)) && aligned(dZ, dtype_bytes(dt)) && aligned(loss, 4) && aligned(weight, 4) &&
                    aligned(logits, 4) && aligned(ids, 8) && aligned(labels, 8) && aligned(status, 4),
                DP_EINVAL);
    const Args a = {V, ids, logits, (int)K, labels, alpha, tau, weight, loss, status};
    return dt == DP_F32 ? run<float>(Z, M, a, dZ, stream) : run<uint16_t>(Z, M, a, dZ, stream);
}
