// The l2 norm of one gradient held in many tensors, and its clipping:
//   norm = sqrt(sum_k sum_e g_k[e]^2),  out_k = min(1, C / (norm + 1e-6)) * g_k
//
// The norm needs every value before the first output can be written, so the
// values are read twice and written once; both passes are bound by those
// bytes.  The tensors are cut into chunks of one size (chosen so that a call
// has about kTargetChunks of them); a workgroup takes one chunk.
// 1. sumsq_kernel: each chunk's sum of squares, in 64 bits, to the workspace;
// 2. norm_kernel: the chunks' sums, added in a fixed order by one workgroup,
//    and the clip factor;
// 3. scale_kernel: the outputs, chunks in descending order, so that what the
//    first pass read last (and the caches still hold) is read first.
// Calls of at most kFoldChunks chunks leave out 2.: every workgroup of 3. adds
// the few sums itself.  Up to kBatch tensors go into a launch.
//
// Squares and sums are in fp64: the vector unit has the rate to spare (a
// conversion and a multiply-add per value, against the 4 bytes that it is
// read from), and no finite value overflows or vanishes when squared.
#include "common.hpp"

namespace dpg {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 96;                // tensors per launch (their table is a kernel argument)
constexpr int kMinChunk = 4096;           // elements
constexpr i64 kTargetChunks = 4096;
constexpr int kFoldChunks = 512;
constexpr int kHeader = 16;               // bytes of the workspace before the chunks' sums
constexpr int kMaxCount = 65536;

struct Batch {
    int count;
    int chunk0;                           // the batch's first chunk among the call's
    int chunks;                           // all chunks of the call
    i64 chunk;                            // elements
    const void *g[kBatch];
    void *out[kBatch];
    i64 numel[kBatch];
    int blk0[kBatch + 1];                 // first workgroup of each tensor in this launch
    uint8_t bf16[kBatch];
};

__device__ __forceinline__ int find_tensor(const Batch &b, int blk)
{
    int lo = 0, hi = b.count;             // blk0[lo] <= blk < blk0[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.blk0[mid] <= blk) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double wave_sum64(double v)
{
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// Sum over the workgroup in a fixed order, valid in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum64(double v, double *red)
{
    v = wave_sum64(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += red[w];
    return s;
}

// sum of p[0 .. n-1], each thread a fixed share, eight loads in flight
template <int THREADS>
__device__ __forceinline__ double sum_chunks(const double *__restrict__ p, int n, double *red)
{
    double s = 0.0;
    for (int k = threadIdx.x; k < n; k += 8 * THREADS) {
        double v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = k + j * THREADS < n ? p[k + j * THREADS] : 0.0;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[j];
    }
    return block_sum64<THREADS>(s, red);
}

template <typename T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
};

__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[4])
{
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[8])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t bf16_bits(float x)
{
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ uint4 pack(const float (&v)[4])
{
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_elem(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(uint16_t *p, float v) { *p = (uint16_t)bf16_bits(v); }

constexpr int kInFlight = 4;              // 16-byte loads of a thread in flight

// elements before the first 16-byte boundary of p, at most n
template <typename T>
__device__ __forceinline__ i64 head_of(const T *p, i64 n)
{
    const i64 h = (i64)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (i64)sizeof(T);
    return h < n ? h : n;
}

template <typename T>
__device__ __forceinline__ double chunk_sumsq(const T *__restrict__ p, i64 n)
{
    constexpr int VN = Vec<T>::N;
    const i64 head = head_of(p, n);
    const i64 nv = (n - head) / VN;
    const uint4 *q = reinterpret_cast<const uint4 *>(p + head);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    i64 i = threadIdx.x;
    for (; i + (kInFlight - 1) * kThreads < nv; i += kInFlight * kThreads) {
        uint4 r[kInFlight];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) r[k] = q[i + k * kThreads];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
            float v[VN];
            unpack(r[k], v);
#pragma unroll
            for (int j = 0; j < VN; ++j) s[j & 3] = fma((double)v[j], (double)v[j], s[j & 3]);
        }
    }
    for (; i < nv; i += kThreads) {
        float v[VN];
        unpack(q[i], v);
#pragma unroll
        for (int j = 0; j < VN; ++j) s[j & 3] = fma((double)v[j], (double)v[j], s[j & 3]);
    }
    // the elements before the first and after the last 16-byte piece (fewer than 2 VN)
    const i64 rest = n - VN * nv;
    if (threadIdx.x < rest) {
        const i64 e = threadIdx.x < head ? threadIdx.x : VN * nv + threadIdx.x;
        const double v = (double)load_elem<T>(p, e);
        s[0] = fma(v, v, s[0]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T *p, T *o, i64 n, float c)
{
    constexpr int VN = Vec<T>::N;
    if (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15) != 0) {
        // no 16-byte boundary in common: by elements
        for (i64 e = threadIdx.x; e < n; e += kThreads) store_elem(o + e, c * load_elem<T>(p, e));
        return;
    }
    const i64 head = head_of(p, n);
    const i64 nv = (n - head) / VN;
    const uint4 *q = reinterpret_cast<const uint4 *>(p + head);
    uint4 *t = reinterpret_cast<uint4 *>(o + head);
    i64 i = threadIdx.x;
    for (; i + (kInFlight - 1) * kThreads < nv; i += kInFlight * kThreads) {
        uint4 r[kInFlight];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) r[k] = q[i + k * kThreads];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) {
            float v[VN];
            unpack(r[k], v);
#pragma unroll
            for (int j = 0; j < VN; ++j) v[j] *= c;
            t[i + k * kThreads] = pack(v);
        }
    }
    for (; i < nv; i += kThreads) {
        float v[VN];
        unpack(q[i], v);
#pragma unroll
        for (int j = 0; j < VN; ++j) v[j] *= c;
        t[i] = pack(v);
    }
    const i64 rest = n - VN * nv;
    if (threadIdx.x < rest) {
        const i64 e = threadIdx.x < head ? threadIdx.x : VN * nv + threadIdx.x;
        store_elem(o + e, c * load_elem<T>(p, e));
    }
}

// the chunk of workgroup blk: its tensor, first element and length
__device__ __forceinline__ int chunk_of(const Batch &b, int blk, i64 &first, i64 &n)
{
    const int k = find_tensor(b, blk);
    first = (i64)(blk - b.blk0[k]) * b.chunk;
    n = b.numel[k] - first < b.chunk ? b.numel[k] - first : b.chunk;
    return k;
}

__global__ __launch_bounds__(kThreads) void sumsq_kernel(Batch b, double *__restrict__ sums)
{
    __shared__ double red[kThreads / 64];
    i64 first, n;
    const int k = chunk_of(b, (int)blockIdx.x, first, n);
    const double s = b.bf16[k] ? chunk_sumsq((const uint16_t *)b.g[k] + first, n)
                               : chunk_sumsq((const float *)b.g[k] + first, n);
    const double t = block_sum64<kThreads>(s, red);
    if (threadIdx.x == 0) sums[b.chunk0 + blockIdx.x] = t;
}

__global__ __launch_bounds__(1024) void norm_kernel(const double *__restrict__ sums, int n, float C,
                                                    float *__restrict__ factor, float *__restrict__ norm,
                                                    int32_t *status)
{
    __shared__ double red[16];
    const double s = sum_chunks<1024>(sums, n, red);
    if (threadIdx.x != 0) return;
    const float v = (float)sqrt(s);
    *norm = v;
    *factor = clip_factor(v, C);
    if (!isfinite(v)) raise_flag(status, DP_FLAG_NONFINITE);
}

// FOLD: the norm and the factor are formed here, from the chunks' sums
template <bool FOLD>
__global__ __launch_bounds__(kThreads) void scale_kernel(Batch b, const double *__restrict__ sums,
                                                         const float *__restrict__ factor, float C,
                                                         float *__restrict__ norm, int32_t *status)
{
    __shared__ double red[kThreads / 64];
    float c;
    if constexpr (FOLD) {
        const float v = (float)sqrt(sum_chunks<kThreads>(sums, b.chunks, red));
        c = clip_factor(v, C);
        if (b.chunk0 == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
            *norm = v;
            if (!isfinite(v)) raise_flag(status, DP_FLAG_NONFINITE);
        }
    } else {
        c = *factor;
    }
    i64 first, n;
    const int k = chunk_of(b, (int)(gridDim.x - 1 - blockIdx.x), first, n);
    if (b.out[k] == nullptr) return;
    if (b.bf16[k]) chunk_scale((const uint16_t *)b.g[k] + first, (uint16_t *)b.out[k] + first, n, c);
    else chunk_scale((const float *)b.g[k] + first, (float *)b.out[k] + first, n, c);
}

// elements per chunk: kMinChunk, doubled until the call has at most kTargetChunks of them (and one per tensor)
i64 chunk_size(const dp_grad_tensor *items, int32_t count)
{
    i64 chunk = kMinChunk;
    for (;; chunk *= 2) {
        i64 n = 0;
        for (int32_t k = 0; k < count; ++k) n += items[k].numel / chunk;
        if (n <= kTargetChunks) return chunk;
    }
}

i64 count_chunks(const dp_grad_tensor *items, int32_t count, i64 chunk)
{
    i64 n = 0;
    for (int32_t k = 0; k < count; ++k) n += ceil_div(items[k].numel, chunk);
    return n;
}

dp_status check(const dp_grad_tensor *items, int32_t count)
{
    DPG_REQUIRE(count >= 0 && count <= kMaxCount && (count == 0 || items != nullptr), DP_EINVAL);
    for (int32_t k = 0; k < count; ++k) {
        DPG_REQUIRE(dtype_ok((dp_dtype)items[k].dtype), DP_EDTYPE);
        DPG_REQUIRE(items[k].numel >= 0 && (items[k].numel == 0 || items[k].g != nullptr), DP_EINVAL);
        const uintptr_t e = dtype_bytes((dp_dtype)items[k].dtype);
        DPG_REQUIRE(aligned(items[k].g, e) && aligned(items[k].out, e), DP_EINVAL);
        DPG_REQUIRE(items[k].numel < (i64(1) << 40), DP_EUNSUPPORTED);
    }
    return DP_OK;
}

}  // namespace
}  // namespace dpg

using namespace dpg;

extern "C" size_t dp_clip_global_norm_many_workspace_bytes(const dp_grad_tensor *items, int32_t count)
{
    if (check(items, count) != DP_OK) return 0;
    return kHeader + sizeof(double) * (size_t)count_chunks(items, count, chunk_size(items, count));
}

extern "C" dp_status dp_clip_global_norm_many(const dp_grad_tensor *items, int32_t count, float C, float *norm,
                                              int32_t *status, void *ws, size_t ws_bytes, hipStream_t stream)
{
    const dp_status bad = check(items, count);
    if (bad != DP_OK) return bad;
    DPG_REQUIRE(C > 0.0f && norm != nullptr, DP_EINVAL);
    const i64 chunk = chunk_size(items, count);
    const int chunks = (int)count_chunks(items, count, chunk);
    DPG_REQUIRE(ws != nullptr && aligned(ws, 16) && ws_bytes >= kHeader + sizeof(double) * (size_t)chunks, DP_EINVAL);
    float *factor = (float *)ws;
    double *sums = (double *)((char *)ws + kHeader);
    bool any_out = false;
    for (int32_t k = 0; k < count; ++k) any_out |= items[k].out != nullptr && items[k].numel > 0;
    const bool fold = any_out && chunks <= kFoldChunks;
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1 && !fold) norm_kernel<<<1, 1024, 0, stream>>>(sums, chunks, C, factor, norm, status);
        if (pass == 1 && !any_out) break;
        int chunk0 = 0;
        Batch b;
        b.count = 0;
        b.blk0[0] = 0;
        b.chunks = chunks;
        b.chunk = chunk;
        for (int32_t k = 0; k <= count; ++k) {
            if (b.count == kBatch || (k == count && b.count > 0)) {
                b.chunk0 = chunk0;
                const int blocks = b.blk0[b.count];
                if (pass == 0) sumsq_kernel<<<(unsigned)blocks, kThreads, 0, stream>>>(b, sums);
                else if (fold)
                    scale_kernel<true><<<(unsigned)blocks, kThreads, 0, stream>>>(b, sums, factor, C, norm, status);
                else scale_kernel<false><<<(unsigned)blocks, kThreads, 0, stream>>>(b, sums, factor, C, norm, status);
                chunk0 += blocks;
                b.count = 0;
            }
            if (k == count) break;
            if (items[k].numel == 0) continue;
            const int j = b.count++;
            b.g[j] = items[k].g;
            b.out[j] = items[k].out;
            b.numel[j] = items[k].numel;
            b.bf16[j] = items[k].dtype == DP_BF16;
            b.blk0[j + 1] = b.blk0[j] + (int)ceil_div(items[k].numel, chunk);
        }
    }
    return launch_status();
}
