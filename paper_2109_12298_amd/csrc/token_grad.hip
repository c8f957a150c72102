// Clipped gradient of an Embedding layer by sorted tokens:
//   sum[v][:] = s * sum over positions m with ids[m] = v of c_n(m) * B[m][:]
//
// 1. The positions are sorted by id (stable, so equal ids keep ascending
//    positions): a least-significant-digit radix sort of (id, position) with
//    digits of up to 9 bits.  A position that is left out (a bad id, a sample
//    outside the active batch) takes the key V and sorts behind all others.
//    - up to kSmallMax positions: one workgroup, all digits in LDS, while the
//      other workgroups of the launch write zeros to all of sum;
//    - beyond: per digit a count launch and a scatter launch.  The first
//      count clears a byte per id, the first scatter sets those of the ids it
//      meets, so that only rows without a token are zeroed (by workgroups of
//      launch 2 that have no rows to add).
// 2. walk_kernel: the sorted positions in chunks; a wave adds a chunk's rows
//    of one block of columns, kBatch row loads in flight, and writes each id's
//    sum where the id's positions start and end inside the chunk.  A piece
//    of an id that crosses chunks goes to the workspace.
// 3. join_kernel: the pieces of such an id in chunk order.
// The order of every sum depends on the ids alone; no atomics touch data.
#include "common.hpp"

#include <type_traits>

namespace dpg {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSmallMax = 8192;           // positions sorted by one workgroup
constexpr int kScanTiles = 64;            // tiles whose counts a scatter workgroup adds up itself
constexpr int kWalkWaves = 4;
constexpr int kWalkThreads = 64 * kWalkWaves;
constexpr int kBatch = 16;                // rows whose loads a wave has in flight
constexpr int kFillRows = 16;             // rows of sum that a zeroing wave looks at together
constexpr int kFillBlocks = 1024;

// Sort tiles are of 1024 * ITEMS positions: few items (little work per
// workgroup) while the tiles are few, more beyond.
int items_for(i64 M) { return M <= (i64)kScanTiles * 2 * kSortThreads ? 2 : 8; }

struct Plan {
    i64 M, tiles, chunk, chunks, colblocks;
    int items, passes, bits, vec;         // bits per digit; columns per lane
    size_t keys[2], pos[2], hist, tot, present, part, bytes;    // workspace offsets
};

Plan make_plan(i64 N, i64 T, i64 V, i64 D, int vec)
{
    Plan p;
    p.M = N * T;
    p.items = items_for(p.M);
    p.tiles = ceil_div(p.M, (i64)p.items * kSortThreads);
    int key_bits = 1;
    while ((V >> key_bits) != 0) ++key_bits;             // keys are 0 .. V
    p.passes = (key_bits + kDigitBits - 1) / kDigitBits;
    p.bits = (key_bits + p.passes - 1) / p.passes;
    p.vec = vec;
    p.colblocks = ceil_div(D, 64 * (i64)vec);
    // chunks of 16 to 256 sorted positions, as long as 4096 waves remain
    p.chunk = 16;
    while (p.chunk < 256 && p.M / (2 * p.chunk) * p.colblocks >= 4096) p.chunk *= 2;
    p.chunks = ceil_div(p.M, p.chunk);
    size_t o = 0;
    const auto take = [&](size_t n) {
        const size_t at = o;
        o += align_up(n, 256);
        return at;
    };
    const bool small = p.M <= kSmallMax;
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = take(i == 0 || !small ? 4 * (size_t)p.M : 0);
        p.pos[i] = take(i == 0 || !small ? 4 * (size_t)p.M : 0);
    }
    p.hist = take(small ? 0 : 4 * (size_t)p.tiles * kDigits);
    p.tot = take(small ? 0 : 4 * (size_t)kDigits);
    p.present = take(small ? 0 : (size_t)V);
    p.part = take(2 * sizeof(float) * (size_t)p.chunks * (size_t)D);
    p.bytes = o;
    return p;
}

// ---------------------------------------------------------------------------
// sort
// ---------------------------------------------------------------------------

// the key of position m: its id, or V if the position is left out
__device__ __forceinline__ uint32_t key_of(const int64_t *ids, uint32_t m, uint32_t T, i64 V, const float *norm,
                                           bool &bad)
{
    if (norm != nullptr && norm[m / T] < 0.0f) return (uint32_t)V;
    const int64_t id = ids[m];
    if (id >= 0 && id < V) return (uint32_t)id;
    bad = true;
    return (uint32_t)V;
}

// Exclusive scan of one int per thread over the workgroup of kSortThreads.
__device__ __forceinline__ int scan_1024(int v, int *wsum)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, kWave);
        if (lane >= o) x += y;
    }
    if (lane == 63) wsum[w] = x;
    __syncthreads();
    int pre = 0;
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) pre += i < w ? wsum[i] : 0;
    __syncthreads();
    return pre + x - v;
}

// Ranks of a tile's items among the items of equal digit: cnt[w][d] is left
// holding, per wave w and digit d, the items of digit d in the waves before w,
// and the total per digit is returned in the thread whose index is the digit.
// Wave w's item i of lane l is the tile's position (w * ITEMS + i) * 64 + l.
template <int ITEMS>
__device__ __forceinline__ int rank_tile(const uint32_t (&digit)[ITEMS], const bool (&on)[ITEMS], int bits,
                                         int (*cnt)[kDigits], int (&rank)[ITEMS])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int i = lane; i < kDigits; i += 64) cnt[w][i] = 0;      // the wave's own row
    const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        uint64_t same = __ballot(on[i]);                         // lanes whose item has this lane's digit
        for (int b = 0; b < bits; ++b) {
            const bool bit = (digit[i] >> b) & 1u;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        rank[i] = 0;
        if (on[i]) {
            const int before = __popcll(same & below);
            const int base = cnt[w][digit[i]];
            rank[i] = base + before;
            if (before == 0) cnt[w][digit[i]] = base + __popcll(same);
        }
    }
    __syncthreads();
    int run = 0;
    if (threadIdx.x < kDigits) {
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const int t = cnt[k][threadIdx.x];
            cnt[k][threadIdx.x] = run;
            run += t;
        }
    }
    return run;
}

// zeros to the 16-byte pieces [lo, hi) of a 16-byte aligned array, by the workgroups first, first + 1, ...
__device__ __forceinline__ void fill16(uint4 *p, i64 n, i64 block, i64 blocks)
{
    const uint4 z = make_uint4(0, 0, 0, 0);
    for (i64 i = block * blockDim.x + threadIdx.x; i < n; i += blocks * blockDim.x) p[i] = z;
}

// The whole sort in workgroup 0; the others write zeros to sum.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void small_sort_kernel(const int64_t *__restrict__ ids, int M, uint32_t T,
                                                                  i64 V, const float *__restrict__ norm, int passes,
                                                                  int bits, uint32_t *__restrict__ keys_out,
                                                                  uint32_t *__restrict__ pos_out,
                                                                  float *__restrict__ sum, i64 sum_n, int32_t *status)
{
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int wsum[kSortWaves];
    __shared__ uint32_t kbuf[ITEMS * kSortThreads], pbuf[ITEMS * kSortThreads];
    if (blockIdx.x > 0) {
        const i64 b = blockIdx.x - 1, nb = gridDim.x - 1;
        if ((reinterpret_cast<uintptr_t>(sum) & 15) == 0) {
            fill16(reinterpret_cast<uint4 *>(sum), sum_n / 4, b, nb);
            if (b == 0 && threadIdx.x < (sum_n & 3)) sum[sum_n - 1 - threadIdx.x] = 0.0f;
        } else {
            for (i64 i = b * blockDim.x + threadIdx.x; i < sum_n; i += nb * blockDim.x) sum[i] = 0.0f;
        }
        return;
    }
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t key[ITEMS], pos[ITEMS], digit[ITEMS];
    bool on[ITEMS], bad = false;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int m = (w * ITEMS + i) * 64 + lane;
        on[i] = m < M;
        pos[i] = (uint32_t)m;
        key[i] = on[i] ? key_of(ids, (uint32_t)m, T, V, norm, bad) : 0;
    }
    if (bad) raise_flag(status, DP_FLAG_BAD_INDEX);
    for (int p = 0; p < passes; ++p) {
        int rank[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) digit[i] = (key[i] >> (p * bits)) & ((1u << bits) - 1u);
        const int total = rank_tile<ITEMS>(digit, on, bits, cnt, rank);
        const int base = scan_1024(total, wsum);
        if (threadIdx.x < kDigits) {
#pragma unroll
            for (int k = 0; k < kSortWaves; ++k) cnt[k][threadIdx.x] += base;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (!on[i]) continue;
            const int at = cnt[w][digit[i]] + rank[i];
            if (p + 1 < passes) {
                kbuf[at] = key[i];
                pbuf[at] = pos[i];
            } else {
                keys_out[at] = key[i];
                pos_out[at] = pos[i];
            }
        }
        if (p + 1 < passes) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int m = (w * ITEMS + i) * 64 + lane;
                if (!on[i]) continue;
                key[i] = kbuf[m];
                pos[i] = pbuf[m];
            }
            __syncthreads();
        }
    }
}

// hist[d][tile] = the tile's keys of digit d.  FIRST: the keys are formed
// here (and kept), and the byte per id is cleared.
template <int ITEMS, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void count_kernel(const int64_t *__restrict__ ids, uint32_t M, uint32_t T,
                                                             i64 V, const float *__restrict__ norm,
                                                             uint32_t *__restrict__ keys, int shift, int bits,
                                                             int32_t *__restrict__ hist, uint8_t *__restrict__ present,
                                                             int32_t *status)
{
    __shared__ int cnt[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) cnt[d] = 0;
    if constexpr (FIRST) fill16(reinterpret_cast<uint4 *>(present), (V + 15) / 16, blockIdx.x, gridDim.x);
    __syncthreads();
    const uint32_t m0 = blockIdx.x * (uint32_t)(ITEMS * kSortThreads);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t m = m0 + i * kSortThreads + threadIdx.x;
        if (m >= M) continue;
        uint32_t k;
        if constexpr (FIRST) {
            k = key_of(ids, m, T, V, norm, bad);
            keys[m] = k;
        } else {
            k = keys[m];
        }
        atomicAdd(&cnt[(k >> shift) & ((1u << bits) - 1u)], 1);
    }
    if (bad) raise_flag(status, DP_FLAG_BAD_INDEX);
    __syncthreads();
    for (int d = threadIdx.x; d < (1 << bits); d += kSortThreads) hist[(i64)d * gridDim.x + blockIdx.x] = cnt[d];
}

// many tiles: hist[d][:] becomes its exclusive prefix sums, tot[d] its sum (one workgroup per digit)
__global__ __launch_bounds__(kSortThreads) void scan_kernel(int32_t *__restrict__ hist, int32_t *__restrict__ tot,
                                                            int tiles)
{
    __shared__ int wsum[kSortWaves];
    __shared__ int last;
    int32_t *h = hist + (i64)blockIdx.x * tiles;
    int carry = 0;
    for (int t0 = 0; t0 < tiles; t0 += kSortThreads) {
        const int t = t0 + threadIdx.x;
        const int v = t < tiles ? h[t] : 0;
        const int e = scan_1024(v, wsum);
        if (t < tiles) h[t] = carry + e;
        if (threadIdx.x == kSortThreads - 1) last = e + v;
        __syncthreads();
        carry += last;
        __syncthreads();
    }
    if (threadIdx.x == 0) tot[blockIdx.x] = carry;
}

// The tile's (key, position) pairs to their places by the digit.  pos_in
// NULL: positions are the indexes (the first digit), and the ids' bytes are set.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void scatter_kernel(const uint32_t *__restrict__ keys_in,
                                                               const uint32_t *__restrict__ pos_in,
                                                               uint32_t *__restrict__ keys_out,
                                                               uint32_t *__restrict__ pos_out, uint32_t M, i64 V,
                                                               int shift, int bits, const int32_t *__restrict__ hist,
                                                               const int32_t *__restrict__ tot,
                                                               uint8_t *__restrict__ present)
{
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int wsum[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int tiles = (int)gridDim.x, tile = (int)blockIdx.x;
    uint32_t key[ITEMS], pos[ITEMS], digit[ITEMS];
    bool on[ITEMS];
    int rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t m = (uint32_t)tile * (ITEMS * kSortThreads) + (w * ITEMS + i) * 64 + lane;
        on[i] = m < M;
        key[i] = on[i] ? keys_in[m] : 0;
        pos[i] = on[i] && pos_in != nullptr ? pos_in[m] : m;
        digit[i] = (key[i] >> shift) & ((1u << bits) - 1u);
    }
    // the items of the thread's digit in all tiles, and in the tiles before this one
    int total = 0, before = 0;
    if (threadIdx.x < (1u << bits)) {
        const int32_t *h = hist + (i64)threadIdx.x * tiles;
        if (tot != nullptr) {
            total = tot[threadIdx.x];
            before = h[tile];
        } else {
            for (int t = 0; t < tiles; t += 8) {
                int v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = t + j < tiles ? h[t + j] : 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    total += v[j];
                    before += t + j < tile ? v[j] : 0;
                }
            }
        }
    }
    rank_tile<ITEMS>(digit, on, bits, cnt, rank);
    const int base = scan_1024(total, wsum) + before;
    if (threadIdx.x < kDigits) {
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) cnt[k][threadIdx.x] += base;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (!on[i]) continue;
        const int at = cnt[w][digit[i]] + rank[i];
        keys_out[at] = key[i];
        pos_out[at] = pos[i];
        if (pos_in == nullptr && key[i] < (uint32_t)V) present[key[i]] = 1;
    }
}

// ---------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Row {
    T v[VEC];
};
template <int VEC>
struct alignas(VEC >= 4 ? 16 : 4 * VEC) Out {
    float v[VEC];
};

__device__ __forceinline__ float as_f32(float x) { return x; }
__device__ __forceinline__ float as_f32(uint16_t x) { return bf16_to_f32(x); }

// Workgroups below walk_blocks add rows; the others write zeros to the rows
// of sum that hold no token (present NULL: they are zero already).
template <typename T, int VEC>
__global__ __launch_bounds__(kWalkThreads) void walk_kernel(
    const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos, const T *__restrict__ B, uint32_t M,
    uint32_t Tn, uint32_t V, i64 D, float scale, const float *__restrict__ norm, float C, uint32_t chunk,
    uint32_t chunks, uint32_t colblocks, uint32_t walk_blocks, float *__restrict__ sum, float *__restrict__ part,
    const uint8_t *__restrict__ present)
{
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= walk_blocks) {
        const uint32_t w0 = (blockIdx.x - walk_blocks) * kWalkWaves + wave;
        const uint32_t nw = (gridDim.x - walk_blocks) * kWalkWaves;
        const uint32_t groups = (V + kFillRows - 1) / kFillRows;
        for (uint32_t g = w0; g < groups; g += nw) {
            const uint32_t v0 = g * kFillRows, v = v0 + lane;
            uint32_t empty = (uint32_t)__ballot(lane < kFillRows && v < V && present[v < V ? v : 0] == 0);
            while (empty != 0) {
                const int j = __ffs((int)empty) - 1;
                empty &= empty - 1;
                float *row = sum + (i64)(v0 + j) * D;
                Out<VEC> z;
#pragma unroll
                for (int i = 0; i < VEC; ++i) z.v[i] = 0.0f;
                for (i64 c = (i64)lane * VEC; c < D; c += 64 * VEC) *reinterpret_cast<Out<VEC> *>(row + c) = z;
            }
        }
        return;
    }
    const uint32_t u = blockIdx.x * kWalkWaves + wave;
    const uint32_t ck = u / colblocks;
    if (ck >= chunks) return;
    const i64 col = (i64)(u % colblocks) * 64 * VEC + lane * VEC;
    const bool on = col < D;
    const T *Bc = B + (on ? col : 0);
    const uint32_t lo = ck * chunk, hi = lo + chunk < M ? lo + chunk : M;
    bool here = lo == 0 || keys[lo - 1] != keys[lo];         // the current id's positions start in this chunk
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    const auto put = [&](float *dst, float f) {
        Out<VEC> o;
#pragma unroll
        for (int i = 0; i < VEC; ++i) o.v[i] = f * acc[i];
        if (on) *reinterpret_cast<Out<VEC> *>(dst + col) = o;
    };
    bool open = false;                                       // the last position's id continues in the next chunk
    for (uint32_t r0 = lo; r0 < hi; r0 += kBatch) {
        // lane l (and l + 16, ...) holds sorted position r0 + l of the batch
        const uint32_t r = r0 + (lane & (kBatch - 1));
        const uint32_t key = r < hi ? keys[r] : V;
        const bool ok = key < V;
        const uint32_t p = ok ? pos[r] : 0;
        const float c = ok && norm != nullptr ? clip_factor(norm[p / Tn], C) : 1.0f;
        const bool ends = ok && (r + 1 >= M || keys[r + 1] != key);
        const uint32_t okm = (uint32_t)__ballot(ok) & ((1u << kBatch) - 1);
        const uint32_t endm = (uint32_t)__ballot(ends);
        if (okm == 0) break;                                 // positions left out sort last
        Row<T, VEC> v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t pj = __builtin_amdgcn_readlane(p, j);
            v[j] = *reinterpret_cast<const Row<T, VEC> *>(Bc + (i64)pj * D);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (((okm >> j) & 1u) == 0) continue;
            const float cj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c), j));
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] = fmaf(cj, as_f32(v[j].v[i]), acc[i]);
            open = true;
            if ((endm >> j) & 1u) {
                if (here) put(sum + (i64)__builtin_amdgcn_readlane(key, j) * D, scale);
                else put(part + (i64)(2 * ck) * D, 1.0f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
                here = true;
                open = false;
            }
        }
    }
    if (open) put(part + (i64)(2 * ck + (here ? 1 : 0)) * D, 1.0f);
}

// Chunk ck's last id, if its positions start in the chunk and continue behind
// it: its piece there, then the following chunks' pieces, added in chunk
// order (each of the four waves a run of them, then the waves in order).
template <int VEC>
__global__ __launch_bounds__(kWalkThreads) void join_kernel(const uint32_t *__restrict__ keys, uint32_t M, uint32_t V,
                                                            i64 D, float scale, uint32_t chunk, uint32_t colblocks,
                                                            float *__restrict__ sum, const float *__restrict__ part)
{
    __shared__ float red[kWalkWaves][64 * VEC];
    const uint32_t ck = blockIdx.x / colblocks;
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lo = ck * chunk, hi = lo + chunk;         // the grid leaves out the last chunk: hi < M
    const uint32_t key = keys[hi - 1];
    if (key >= V || keys[hi] != key || (lo > 0 && keys[lo - 1] == key)) return;
    // the following chunks that hold the id up to their end and behind it
    uint32_t n = 0;
    for (;;) {
        const uint32_t h = (ck + 2 + n + lane) * chunk;      // end of chunk ck + 1 + n + lane
        const bool full = h < M && keys[h - 1] == key && keys[h] == key;
        const uint64_t stop = ~__ballot(full);
        if (stop != 0) {
            n += __ffsll((unsigned long long)stop) - 1;
            break;
        }
        n += 64;
    }
    ++n;                                                     // and the one in which it ends
    const i64 col = (i64)(blockIdx.x % colblocks) * 64 * VEC + lane * VEC;
    const bool on = col < D;
    const float *P = part + (i64)(2 * (ck + 1)) * D + (on ? col : 0);
    const uint32_t per = (n + kWalkWaves - 1) / kWalkWaves;
    const uint32_t x0 = wave * per < n ? wave * per : n, x1 = x0 + per < n ? x0 + per : n;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    if (wave == 0) {
        const Out<VEC> o = *reinterpret_cast<const Out<VEC> *>(part + (i64)(2 * ck + 1) * D + (on ? col : 0));
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = o.v[i];
    }
    for (uint32_t x = x0; x < x1; x += 8) {
        Out<VEC> v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = *reinterpret_cast<const Out<VEC> *>(P + (i64)(2 * (x + j < x1 ? x + j : x)) * D);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (x + j < x1) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] += v[j].v[i];
            }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) red[wave][VEC * lane + i] = acc[i];
    __syncthreads();
    if (wave != 0 || !on) return;
    Out<VEC> o;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        float s = acc[i];
#pragma unroll
        for (int w = 1; w < kWalkWaves; ++w) s += red[w][VEC * lane + i];
        o.v[i] = scale * s;
    }
    *reinterpret_cast<Out<VEC> *>(sum + (i64)key * D + col) = o;
}

// Columns per lane: the fewest that let 64 lanes cover a row, as far as every
// row start of B and sum is aligned for them (16-byte loads at most).
int vec_for(const void *B, const float *sum, dp_dtype dt, i64 D)
{
    const int most = dt == DP_F32 ? 4 : 8;
    int vec = 1;
    while (vec < most && 64 * (i64)vec < D) vec *= 2;
    const auto fits = [&](int v) {
        return D % v == 0 && aligned(B, (uintptr_t)(v * dtype_bytes(dt))) && aligned(sum, v >= 4 ? 16 : 4 * v);
    };
    while (vec > 1 && !fits(vec)) vec /= 2;
    return vec;
}

template <typename T, int VEC>
void sums(const Plan &p, const void *B, i64 T_, i64 V, i64 D, float scale, const float *norm, float C, float *sum,
          char *ws, int buf, hipStream_t stream)
{
    const uint32_t *keys = (const uint32_t *)(ws + p.keys[buf]), *pos = (const uint32_t *)(ws + p.pos[buf]);
    float *part = (float *)(ws + p.part);
    const bool small = p.M <= kSmallMax;
    const uint32_t walk_blocks = (uint32_t)ceil_div(p.chunks * p.colblocks, kWalkWaves);
    const i64 fill = small ? 0 : ceil_div(ceil_div(V, kFillRows), kWalkWaves);
    const uint32_t blocks = walk_blocks + (uint32_t)(fill < kFillBlocks ? fill : kFillBlocks);
    walk_kernel<T, VEC><<<blocks, kWalkThreads, 0, stream>>>(
        keys, pos, (const T *)B, (uint32_t)p.M, (uint32_t)T_, (uint32_t)V, D, scale, norm, C, (uint32_t)p.chunk,
        (uint32_t)p.chunks, (uint32_t)p.colblocks, walk_blocks, sum, part,
        small ? nullptr : (const uint8_t *)(ws + p.present));
    if (p.chunks > 1)
        join_kernel<VEC><<<(unsigned)((p.chunks - 1) * p.colblocks), kWalkThreads, 0, stream>>>(
            keys, (uint32_t)p.M, (uint32_t)V, D, scale, (uint32_t)p.chunk, (uint32_t)p.colblocks, sum, part);
}

template <typename T>
void sums_by_vec(const Plan &p, const void *B, i64 T_, i64 V, i64 D, float scale, const float *norm, float C,
                 float *sum, char *ws, int buf, hipStream_t stream)
{
    if (p.vec == 8) {
        if constexpr (std::is_same<T, uint16_t>::value)
            sums<T, 8>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, stream);
    } else if (p.vec == 4) {
        sums<T, 4>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, stream);
    } else if (p.vec == 2) {
        sums<T, 2>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, stream);
    } else {
        sums<T, 1>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, stream);
    }
}

// Sorts the positions; returns which of the two buffers holds the result.
template <int ITEMS>
int sort(const Plan &p, const int64_t *ids, i64 T, i64 V, const float *norm, int32_t *status, char *ws,
         hipStream_t stream)
{
    int32_t *hist = (int32_t *)(ws + p.hist);
    int32_t *tot = p.tiles > kScanTiles ? (int32_t *)(ws + p.tot) : nullptr;
    uint8_t *present = (uint8_t *)(ws + p.present);
    const unsigned tiles = (unsigned)p.tiles;
    int buf = 0;
    for (int i = 0; i < p.passes; ++i, buf ^= 1) {
        uint32_t *ki = (uint32_t *)(ws + p.keys[buf]), *ko = (uint32_t *)(ws + p.keys[buf ^ 1]);
        uint32_t *pi = (uint32_t *)(ws + p.pos[buf]), *po = (uint32_t *)(ws + p.pos[buf ^ 1]);
        if (i == 0)
            count_kernel<ITEMS, true><<<tiles, kSortThreads, 0, stream>>>(ids, (uint32_t)p.M, (uint32_t)T, V, norm, ki,
                                                                         0, p.bits, hist, present, status);
        else
            count_kernel<ITEMS, false><<<tiles, kSortThreads, 0, stream>>>(ids, (uint32_t)p.M, (uint32_t)T, V, norm, ki,
                                                                          i * p.bits, p.bits, hist, present, status);
        if (tot != nullptr) scan_kernel<<<1u << p.bits, kSortThreads, 0, stream>>>(hist, tot, (int)p.tiles);
        scatter_kernel<ITEMS><<<tiles, kSortThreads, 0, stream>>>(ki, i == 0 ? nullptr : pi, ko, po, (uint32_t)p.M, V,
                                                                  i * p.bits, p.bits, hist, tot, present);
    }
    return buf;
}

}  // namespace
}  // namespace dpg

using namespace dpg;

namespace {

dp_status check_sizes(i64 N, i64 T, i64 V, i64 D)
{
    DPG_REQUIRE(N >= 0 && T >= 0 && V >= 1 && D >= 1, DP_EINVAL);
    DPG_REQUIRE(V < (i64(1) << 31), DP_EINVAL);
    // 32-bit sorted positions, with room for a chunk past the last one
    DPG_REQUIRE(N < (i64(1) << 30) && T < (i64(1) << 30) && N * T < (i64(1) << 30), DP_EUNSUPPORTED);
    DPG_REQUIRE(D < (i64(1) << 22), DP_EUNSUPPORTED);
    // a grid holds fewer than 2^24 workgroups of 256: one per 256 positions and 64 columns at the most
    DPG_REQUIRE(N * T * D < (i64(1) << 37), DP_EUNSUPPORTED);
    return DP_OK;
}

}  // namespace

extern "C" size_t dp_clip_accumulate_tokens_workspace_bytes(int64_t N, int64_t T, int64_t V, int64_t D, dp_dtype dt)
{
    if (!dtype_ok(dt) || check_sizes(N, T, V, D) != DP_OK || N * T == 0) return 0;
    // the columns per lane depend on the arrays' alignment too: the largest need over them
    size_t most = 0;
    for (int vec = 1; vec <= (dt == DP_F32 ? 4 : 8); vec *= 2) {
        const size_t b = make_plan(N, T, V, D, vec).bytes;
        most = b > most ? b : most;
    }
    return most;
}

extern "C" dp_status dp_clip_accumulate_tokens(const int64_t *ids, const void *B, dp_dtype dt, int64_t N, int64_t T,
                                               int64_t V, int64_t D, float scale, const float *norm, float C,
                                               float *sum, int32_t *status, void *ws, size_t ws_bytes,
                                               hipStream_t stream)
{
    DPG_REQUIRE(dtype_ok(dt), DP_EDTYPE);
    const dp_status bad = check_sizes(N, T, V, D);
    if (bad != DP_OK) return bad;
    DPG_REQUIRE(sum != nullptr, DP_EINVAL);
    DPG_REQUIRE(norm == nullptr || C > 0.0f, DP_EINVAL);
    if (N * T == 0) {
        zero_fill(sum, V * D, stream);
        return launch_status();
    }
    DPG_REQUIRE(ids != nullptr && B != nullptr, DP_EINVAL);
    const size_t need = dp_clip_accumulate_tokens_workspace_bytes(N, T, V, D, dt);
    DPG_REQUIRE(ws != nullptr && aligned(ws, 16) && ws_bytes >= need, DP_EINVAL);
    const Plan p = make_plan(N, T, V, D, vec_for(B, sum, dt, D));
    char *w = (char *)ws;
    int buf = 0;
    if (p.M <= kSmallMax) {
        const i64 fill = ceil_div(V * D, 16 * kSortThreads);
        const unsigned blocks = 1 + (unsigned)(fill < kFillBlocks ? fill : kFillBlocks);
        uint32_t *keys = (uint32_t *)(w + p.keys[0]), *pos = (uint32_t *)(w + p.pos[0]);
        if (p.M <= 2 * kSortThreads)
            small_sort_kernel<2><<<blocks, kSortThreads, 0, stream>>>(ids, (int)p.M, (uint32_t)T, V, norm, p.passes,
                                                                      p.bits, keys, pos, sum, V * D, status);
        else
            small_sort_kernel<8><<<blocks, kSortThreads, 0, stream>>>(ids, (int)p.M, (uint32_t)T, V, norm, p.passes,
                                                                      p.bits, keys, pos, sum, V * D, status);
    } else {
        buf = p.items == 2 ? sort<2>(p, ids, T, V, norm, status, w, stream)
                           : sort<8>(p, ids, T, V, norm, status, w, stream);
    }
    if (dt == DP_F32) sums_by_vec<float>(p, B, T, V, D, scale, norm, C, sum, w, buf, stream);
    else sums_by_vec<uint16_t>(p, B, T, V, D, scale, norm, C, sum, w, buf, stream);
    return launch_status();
}
