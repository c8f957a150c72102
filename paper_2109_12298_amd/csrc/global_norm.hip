// The l2 norm of one gradient held in many tensors, and its clipping:
//   norm = sqrt(sum_k sum_e g_k[e]^2),  out_k = min(1, C / (norm + 1e-6)) * g_k
//
// The norm needs every value before the first output can be written, so the
// values are read twice and written once; both passes are bound by those
// bytes.  The tensors are cut into chunks of one size (chunk_size); a
// workgroup takes one chunk.
// 1. sumsq_kernel: each chunk's sum of squares, in 64 bits, to the workspace;
// 2. norm_kernel: the chunks' sums, added in a fixed order by one workgroup,
//    and the clip factor;
// 3. scale_kernel: the outputs, chunks in descending order, so that what the
//    caches still hold of the first pass is read first.
// Calls of more than kCachedBytes load and store past the caches, and have
// shorter chunks (fp32, cached and streamed): 37 MB 24 and 27 us, 75 MB 42.5
// and 44, 150 MB 93 and 80, 1.3 GB (4.0 GB moved) 750 and 694, of which the
// first pass takes 206 (6.5 TB/s) and the second, reading and writing, 485.
// Calls of at most kFoldChunks chunks leave out 2.: every workgroup of 3. adds
// the few sums itself.  Up to kBatch tensors go into a launch.  Calls of a few
// tens of thousands of values are one launch of one workgroup (tiny_kernel),
// which keeps them in registers.
//
// Squares and sums are in fp64: the vector unit has the rate to spare (a
// conversion and a multiply-add per value, against the 4 bytes that it is
// read from), and no finite value overflows or vanishes when squared.
#include "common.hpp"

namespace dpg {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 128;               // tensors per launch (their table is a kernel argument)
constexpr int kMinChunk = 4096;           // elements
constexpr int kMidChunk = 32768, kStreamChunk = 8192;
constexpr i64 kMostChunks = 16384;
constexpr int kFoldChunks = 512;
constexpr i64 kCachedBytes = i64(96) << 20;
constexpr int kTinyChunk = 1024;          // elements of a wave's turn in tiny_kernel
constexpr int kTinyTurns = 4;
constexpr int kTinyChunks = 16 * kTinyTurns;
constexpr int kHeader = 16;               // bytes of the workspace before the chunks' sums
constexpr int kMaxCount = 65536;

struct Batch {
    int count;
    int chunk0;                           // the batch's first chunk among the call's
    int chunks;                           // all chunks of the call
    int stream;                           // loads and stores past the caches
    i64 chunk;                            // elements
    const void *g[kBatch];
    void *out[kBatch];
    i64 numel[kBatch];                    // times two, plus one for bf16
    int blk0[kBatch + 1];                 // first workgroup of each tensor in this launch
};
// (No array of bytes or half words in a kernel argument beside pointers:
// scalar loads drop the low bits of both parts of their address, and the
// compiler has been seen to reuse such an array's address as one part of a
// pointer's.)

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

constexpr int kInFlight = 8;              // 16-byte loads of a thread in flight

template <bool STREAM>
__device__ __forceinline__ uint4 load16(const uint4 *p)
{
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    if constexpr (STREAM) {
        const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    return *p;
}

template <bool STREAM>
__device__ __forceinline__ void store16(uint4 *p, const uint4 &v)
{
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    if constexpr (STREAM) __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_t *>(p));
    else *p = v;
}

// elements before the first 16-byte boundary of p, at most n
template <typename T>
__device__ __forceinline__ i64 head_of(const T *p, i64 n)
{
    const i64 h = (i64)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (i64)sizeof(T);
    return h < n ? h : n;
}

template <bool STREAM, typename T>
__device__ __forceinline__ double chunk_sumsq(const T *__restrict__ p, i64 n)
{
    constexpr int VN = Vec<T>::N;
    const i64 head = head_of(p, n);
    const i64 nv = (n - head) / VN;
    const uint4 *q = reinterpret_cast<const uint4 *>(p + head);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    const auto add = [&](const uint4 &r) {
        float v[VN];
        unpack(r, v);
#pragma unroll
        for (int j = 0; j < VN; ++j) s[j & 3] = fma((double)v[j], (double)v[j], s[j & 3]);
    };
    i64 i = threadIdx.x;
    uint4 r[kInFlight];
    for (; i + (kInFlight - 1) * kThreads < nv; i += kInFlight * kThreads) {
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) r[k] = load16<STREAM>(q + i + k * kThreads);
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) add(r[k]);
    }
    if (i < nv) {                         // what is left, all in flight too
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) r[k] = load16<STREAM>(q + (i + k * kThreads < nv ? i + k * kThreads : i));
#pragma unroll
        for (int k = 0; k < kInFlight; ++k)
            if (i + k * kThreads < nv) add(r[k]);
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

template <bool STREAM, typename T>
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
    const auto put = [&](i64 at, const uint4 &r) {
        float v[VN];
        unpack(r, v);
#pragma unroll
        for (int j = 0; j < VN; ++j) v[j] *= c;
        store16<STREAM>(t + at, pack(v));
    };
    i64 i = threadIdx.x;
    uint4 r[kInFlight];
    for (; i + (kInFlight - 1) * kThreads < nv; i += kInFlight * kThreads) {
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) r[k] = load16<STREAM>(q + i + k * kThreads);
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) put(i + k * kThreads, r[k]);
    }
    if (i < nv) {
#pragma unroll
        for (int k = 0; k < kInFlight; ++k) r[k] = load16<STREAM>(q + (i + k * kThreads < nv ? i + k * kThreads : i));
#pragma unroll
        for (int k = 0; k < kInFlight; ++k)
            if (i + k * kThreads < nv) put(i + k * kThreads, r[k]);
    }
    const i64 rest = n - VN * nv;
    if (threadIdx.x < rest) {
        const i64 e = threadIdx.x < head ? threadIdx.x : VN * nv + threadIdx.x;
        store_elem(o + e, c * load_elem<T>(p, e));
    }
}

// the chunk of workgroup blk: its tensor, first element, length and type
__device__ __forceinline__ int chunk_of(const Batch &b, int blk, i64 &first, i64 &n, bool &bf16)
{
    const int k = find_tensor(b, blk);
    const i64 numel = b.numel[k] >> 1;
    bf16 = (b.numel[k] & 1) != 0;
    first = (i64)(blk - b.blk0[k]) * b.chunk;
    n = numel - first < b.chunk ? numel - first : b.chunk;
    return k;
}

__global__ __launch_bounds__(kThreads) void sumsq_kernel(Batch b, double *__restrict__ sums)
{
    __shared__ double red[kThreads / 64];
    i64 first, n;
    bool bf16;
    const int k = chunk_of(b, (int)blockIdx.x, first, n, bf16);
    double s;
    if (bf16) {
        const uint16_t *p = (const uint16_t *)b.g[k] + first;
        s = b.stream ? chunk_sumsq<true>(p, n) : chunk_sumsq<false>(p, n);
    } else {
        const float *p = (const float *)b.g[k] + first;
        s = b.stream ? chunk_sumsq<true>(p, n) : chunk_sumsq<false>(p, n);
    }
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
    bool bf16;
    const int k = chunk_of(b, (int)(gridDim.x - 1 - blockIdx.x), first, n, bf16);
    if (b.out[k] == nullptr) return;
    if (bf16) {
        const uint16_t *p = (const uint16_t *)b.g[k] + first;
        uint16_t *o = (uint16_t *)b.out[k] + first;
        if (b.stream) chunk_scale<true>(p, o, n, c);
        else chunk_scale<false>(p, o, n, c);
    } else {
        const float *p = (const float *)b.g[k] + first;
        float *o = (float *)b.out[k] + first;
        if (b.stream) chunk_scale<true>(p, o, n, c);
        else chunk_scale<false>(p, o, n, c);
    }
}

// A wave's chunk: its values (loads of clamped addresses, so that none waits
// for another), or c times them to their places.
template <typename T>
__device__ __forceinline__ void tiny_load(const T *__restrict__ p, i64 n, float (&v)[kTinyChunk / 64])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kTinyChunk / 64; ++j) v[j] = load_elem<T>(p, lane + 64 * j < n ? lane + 64 * j : 0);
#pragma unroll
    for (int j = 0; j < kTinyChunk / 64; ++j) v[j] = lane + 64 * j < n ? v[j] : 0.0f;
}

template <typename T>
__device__ __forceinline__ void tiny_store(T *__restrict__ o, i64 n, float c, const float (&v)[kTinyChunk / 64])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kTinyChunk / 64; ++j)
        if (lane + 64 * j < n) store_elem(o + lane + 64 * j, c * v[j]);
}

// The whole call in one workgroup: wave w takes chunks w, w + 16, ... of up to
// kTinyChunk elements of one tensor, loaded once by single elements (any
// alignment).
struct Tiny {
    int chunks;
    struct {
        const void *g;
        void *out;
        int32_t n, bf16;
    } at[kTinyChunks];
};

__global__ __launch_bounds__(1024) void tiny_kernel(Tiny b, float C, float *__restrict__ norm, int32_t *status)
{
    __shared__ double red[16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float v[kTinyTurns][kTinyChunk / 64];
#pragma unroll
    for (int t = 0; t < kTinyTurns; ++t) {
        const int k = wave + 16 * t;
        if (k >= b.chunks) continue;
        if (b.at[k].bf16) tiny_load((const uint16_t *)b.at[k].g, b.at[k].n, v[t]);
        else tiny_load((const float *)b.at[k].g, b.at[k].n, v[t]);
    }
    double s = 0.0;
#pragma unroll
    for (int t = 0; t < kTinyTurns; ++t)
        if (wave + 16 * t < b.chunks)
#pragma unroll
            for (int j = 0; j < kTinyChunk / 64; ++j) s = fma((double)v[t][j], (double)v[t][j], s);
    const float x = (float)sqrt(block_sum64<1024>(s, red));
    const float c = clip_factor(x, C);
    if (threadIdx.x == 0) {
        *norm = x;
        if (!isfinite(x)) raise_flag(status, DP_FLAG_NONFINITE);
    }
#pragma unroll
    for (int t = 0; t < kTinyTurns; ++t) {
        const int k = wave + 16 * t;
        if (k >= b.chunks || b.at[k].out == nullptr) continue;
        if (b.at[k].bf16) tiny_store((uint16_t *)b.at[k].out, b.at[k].n, c, v[t]);
        else tiny_store((float *)b.at[k].out, b.at[k].n, c, v[t]);
    }
}

bool streamed(const dp_grad_tensor *items, int32_t count)
{
    i64 bytes = 0;
    for (int32_t k = 0; k < count; ++k) bytes += items[k].numel * (i64)dtype_bytes((dp_dtype)items[k].dtype);
    return bytes > kCachedBytes;
}

// Elements per chunk: doubled from kMinChunk up to a size for the workgroups'
// loads (kMidChunk, kStreamChunk) while there are more than kFoldChunks of
// them, and beyond it while there are more than kMostChunks (and one per
// tensor).
i64 chunk_size(const dp_grad_tensor *items, int32_t count)
{
    const int mid = streamed(items, count) ? kStreamChunk : kMidChunk;
    i64 chunk = kMinChunk;
    for (;; chunk *= 2) {
        i64 n = 0;
        for (int32_t k = 0; k < count; ++k) n += items[k].numel / chunk;
        if (n <= (chunk < mid ? (i64)kFoldChunks : kMostChunks)) return chunk;
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
    const auto add = [](Batch &b, const dp_grad_tensor &x) {
        const int j = b.count++;
        b.g[j] = x.g;
        b.out[j] = x.out;
        b.numel[j] = 2 * x.numel + (x.dtype == DP_BF16 ? 1 : 0);
        b.blk0[j + 1] = b.blk0[j] + (int)ceil_div(x.numel, b.chunk);
    };
    Batch b;
    b.count = 0;
    b.blk0[0] = 0;
    b.chunk0 = 0;
    bool any_out = false;
    i64 tiny = 0;
    for (int32_t k = 0; k < count; ++k) {
        any_out |= items[k].out != nullptr && items[k].numel > 0;
        tiny += ceil_div(items[k].numel, kTinyChunk);
    }
    if (tiny <= kTinyChunks) {
        Tiny t;
        t.chunks = 0;
        for (int32_t k = 0; k < count; ++k)
            for (i64 first = 0; first < items[k].numel; first += kTinyChunk) {
                const i64 left = items[k].numel - first, off = first * (i64)dtype_bytes((dp_dtype)items[k].dtype);
                const int j = t.chunks++;
                t.at[j].g = (const char *)items[k].g + off;
                t.at[j].out = items[k].out != nullptr ? (char *)items[k].out + off : nullptr;
                t.at[j].n = (int32_t)(left < kTinyChunk ? left : kTinyChunk);
                t.at[j].bf16 = items[k].dtype == DP_BF16;
            }
        tiny_kernel<<<1, 1024, 0, stream>>>(t, C, norm, status);
        return launch_status();
    }
    b.chunks = chunks;
    b.chunk = chunk;
    b.stream = streamed(items, count);
    const bool fold = any_out && chunks <= kFoldChunks;
    // 1. over the tensors in order, in batches
    for (int32_t k = 0; k <= count; ++k) {
        if (b.count == kBatch || (k == count && b.count > 0)) {
            sumsq_kernel<<<(unsigned)b.blk0[b.count], kThreads, 0, stream>>>(b, sums);
            b.chunk0 += b.blk0[b.count];
            b.count = 0;
        }
        if (k < count && items[k].numel > 0) add(b, items[k]);
    }
    // 2.
    if (!fold) norm_kernel<<<1, 1024, 0, stream>>>(sums, chunks, C, factor, norm, status);
    if (!any_out) return launch_status();
    // 3. over batches of the tensors from the last one back
    int end = chunks;                     // chunks of the tensors not yet taken
    for (int32_t hi = count; hi > 0;) {
        int32_t lo = hi;
        int n = 0;
        while (lo > 0 && n < kBatch) n += items[--lo].numel > 0;
        b.count = 0;
        for (int32_t k = lo; k < hi; ++k)
            if (items[k].numel > 0) add(b, items[k]);
        hi = lo;
        if (b.count == 0) continue;
        end -= b.blk0[b.count];
        b.chunk0 = end;
        const unsigned blocks = (unsigned)b.blk0[b.count];
        if (fold) scale_kernel<true><<<blocks, kThreads, 0, stream>>>(b, sums, factor, C, norm, status);
        else scale_kernel<false><<<blocks, kThreads, 0, stream>>>(b, sums, factor, C, norm, status);
    }
    return launch_status();
}
