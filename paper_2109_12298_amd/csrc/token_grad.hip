// Clipped gradient of an Embedding layer by sorted tokens:
//   sum[v][:] = s * sum over positions m with ids[m] = v of c_n(m) * B[m][:]
//
// Few positions (one_rule): one launch (one_kernel, below).  Beyond:
// 1. The positions are sorted by id (stable, so equal ids keep ascending
//    positions; a position that is left out, for a bad id or a sample outside
//    the active batch, takes the key V and stands last).  Up to kGroupMax of
//    them in one launch (group_kernel), more by a least-significant-digit
//    radix sort of (id, position) with digits of up to 9 bits, per digit a
//    count launch and a scatter launch.  For a large table the first count
//    clears a byte per id and the first scatter sets those of the ids it
//    meets, so that only rows without a token are zeroed, by workgroups that
//    the launches after it have to spare.
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
constexpr int kOneMax = 2048;             // positions of the one-launch path
constexpr int kOneIds = 16384;            // ids of one of its workgroups, at most
constexpr int kPosBits = 11;
constexpr int kOneItems = kOneMax / kSortThreads;
constexpr int kGroupMax = 16384;          // positions that one launch sorts
constexpr int kGroups = 128;              // its workgroups
constexpr int kGroupPosBits = 14;
constexpr int kGroupItems = kGroupMax / kSortThreads;
constexpr i64 kGroupIds = i64(1) << 24;   // ids it sorts, at most
constexpr int kCompareMax = 128;          // kept positions ranked by comparing each with each
static_assert(kOneMax == 1 << kPosBits && kOneIds <= 1 << (32 - kPosBits - 1), "(id, position) in 31 bits");
static_assert(kGroupMax == 1 << kGroupPosBits && kGroupIds / kGroups <= 1 << (32 - kGroupPosBits - 1), "likewise");
constexpr int kScanTiles = 64;            // tiles whose counts a scatter workgroup adds up itself
constexpr i64 kFillBytes = i64(48) << 20; // zeros that a launch bound by latency writes beside its work
constexpr i64 kFillAllBytes = i64(128) << 20;
constexpr int kWalkWaves = 4;
constexpr int kWalkThreads = 64 * kWalkWaves;
constexpr int kBatch = 16;                // rows whose loads a wave has in flight
constexpr int kFillRows = 2;              // rows of sum that a zeroing wave looks at together
constexpr int kFillBlocks = 1024;

// Sort tiles are of 1024 * ITEMS positions: few items (little work per
// workgroup) while the tiles are few, more beyond.
int items_for(i64 M) { return M <= (i64)kScanTiles * 2 * kSortThreads ? 2 : 8; }

struct Plan {
    i64 M, tiles, hist_ld, chunk, chunks, colblocks;
    int items, passes, bits, vec;         // bits per digit; columns per lane
    bool grouped;                         // sorted in one launch
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
    // (ids of one digit take two launches by digits, and a large table is better zeroed beside more launches: 16384
    // positions of 500 x 4096 48.0 us by digits, 49.7 grouped; 50000 x 1024 69.7 and 73.9)
    p.grouped = p.M <= kGroupMax && V <= kGroupIds && p.passes > 1 && 4 * V * D <= kFillAllBytes;
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
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = take(4 * (size_t)p.M);
        p.pos[i] = take(4 * (size_t)p.M);
    }
    p.hist_ld = p.tiles > kScanTiles ? p.tiles : kScanTiles;
    p.hist = take(4 * (size_t)p.hist_ld * kDigits);
    p.tot = take(4 * (size_t)kDigits);
    p.present = take((size_t)V);
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

// zeros to the n 16-byte pieces at p, of which `blocks` workgroups take equal shares (this one is number `block`)
__device__ __forceinline__ void fill16(uint4 *p, i64 n, i64 block, i64 blocks)
{
    const uint4 z = make_uint4(0, 0, 0, 0);
    for (i64 i = block * blockDim.x + threadIdx.x; i < n; i += blocks * blockDim.x) p[i] = z;
}

// Zeros to the rows of sum whose ids hold no token (present[v] == 0; present
// NULL: to every row), rows in groups of kFillRows, groups [g0, g1): wave w0
// of nw takes groups g0 + w0, + nw, ...
struct Fill {
    float *sum;
    const uint8_t *present;
    uint32_t V, g0, g1;
    i64 D;
};

// (STREAM: stored past the caches)
template <bool STREAM>
__device__ __forceinline__ void fill_rows_as(const Fill &f, uint32_t w0, uint32_t nw)
{
    const int lane = threadIdx.x & 63;
    const bool wide = f.D % 4 == 0 && (reinterpret_cast<uintptr_t>(f.sum) & 15) == 0;
    for (uint32_t g = f.g0 + w0; g < f.g1; g += nw) {
        const uint32_t v0 = g * kFillRows, v = v0 + lane;
        uint32_t empty = (uint32_t)__ballot(lane < kFillRows && v < f.V && (f.present == nullptr || f.present[v] == 0));
        while (empty != 0) {
            const int j = __ffs((int)empty) - 1;
            empty &= empty - 1;
            float *row = f.sum + (i64)(v0 + j) * f.D;
            if (wide) {
                for (i64 c = 4 * lane; c < f.D; c += 256) {
                    if constexpr (STREAM) store_stream4(row + c, 0.0f, 0.0f, 0.0f, 0.0f);
                    else *reinterpret_cast<float4 *>(row + c) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
            } else {
                for (i64 c = lane; c < f.D; c += 64) row[c] = 0.0f;
            }
        }
    }
}

// tables large enough for the flags are larger than the caches
__device__ __forceinline__ void fill_rows(const Fill &f, uint32_t w0, uint32_t nw)
{
    if (f.present != nullptr) fill_rows_as<true>(f, w0, nw);
    else fill_rows_as<false>(f, w0, nw);
}

// hist[d][tile] = the tile's keys of digit d.  FIRST: the keys are formed
// here (and kept), and the byte per id is cleared.  Workgroups past the tiles
// write zeros.
template <int ITEMS, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void count_kernel(const int64_t *__restrict__ ids, uint32_t M, uint32_t T,
                                                             i64 V, const float *__restrict__ norm,
                                                             uint32_t *__restrict__ keys, int shift, int bits,
                                                             int32_t *__restrict__ hist, int tiles, i64 hist_ld,
                                                             uint8_t *__restrict__ present, int32_t *status, Fill fill)
{
    __shared__ int cnt[kDigits];
    if ((int)blockIdx.x >= tiles) {
        fill_rows(fill, (blockIdx.x - tiles) * kSortWaves + (threadIdx.x >> 6), (gridDim.x - tiles) * kSortWaves);
        return;
    }
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) cnt[d] = 0;
    if (FIRST && present != nullptr) fill16(reinterpret_cast<uint4 *>(present), (V + 15) / 16, blockIdx.x, tiles);
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
    for (int d = threadIdx.x; d < (1 << bits); d += kSortThreads) hist[(i64)d * hist_ld + blockIdx.x] = cnt[d];
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
// NULL: positions are the indexes (the first digit), and the ids' bytes are
// set.  Workgroups past the tiles write zeros.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void scatter_kernel(const uint32_t *__restrict__ keys_in,
                                                               const uint32_t *__restrict__ pos_in,
                                                               uint32_t *__restrict__ keys_out,
                                                               uint32_t *__restrict__ pos_out, uint32_t M, i64 V,
                                                               int shift, int bits, const int32_t *__restrict__ hist,
                                                               const int32_t *__restrict__ tot, int tiles, i64 hist_ld,
                                                               uint8_t *__restrict__ present, Fill fill)
{
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int wsum[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int tile = (int)blockIdx.x;
    if (tile >= tiles) {
        fill_rows(fill, (tile - tiles) * kSortWaves + w, (gridDim.x - tiles) * kSortWaves);
        return;
    }
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
        const int32_t *h = hist + (i64)threadIdx.x * hist_ld;
        if (tot != nullptr) {
            total = tot[threadIdx.x];
            before = h[tile];
        } else {                          // at most kScanTiles counts, their loads all in flight
            int4 v[kScanTiles / 4];
#pragma unroll
            for (int j = 0; j < kScanTiles / 4; ++j)
                v[j] = 4 * j < tiles ? *reinterpret_cast<const int4 *>(h + 4 * j) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < kScanTiles / 4; ++j) {
                const int c[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    total += 4 * j + i < tiles ? c[i] : 0;
                    before += 4 * j + i < tile ? c[i] : 0;
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
        if (pos_in == nullptr && present != nullptr && key[i] < (uint32_t)V) present[key[i]] = 1;
    }
}

// The n keys (id, position) of list, kept in ascending position, grouped by the
// digit of their id at `shift` (stable), in place: per-wave counts of each digit,
// prefixes over the waves and the digits.
template <int ITEMS, int POS_BITS>
__device__ __forceinline__ void group_list(uint32_t *list, int n, int shift, int bits, int (*cnt)[kDigits], int *wsum)
{
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rounds = (n + 64 * kSortWaves - 1) / (64 * kSortWaves);       // of each wave, on consecutive keys
    const uint64_t below = (uint64_t(1) << lane) - 1;
    for (int i = lane; i < kDigits; i += 64) cnt[wave][i] = 0;
    uint32_t key[ITEMS];
    int rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (i >= rounds) continue;
        const int e = (wave * rounds + i) * 64 + lane;
        const bool on = e < n;
        key[i] = on ? list[e] : 0;
        const uint32_t d = (key[i] >> (POS_BITS + shift)) & ((1u << bits) - 1u);
        uint64_t same = __ballot(on);
        for (int b = 0; b < bits; ++b) {
            const bool bit = (d >> b) & 1u;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        rank[i] = 0;
        if (on) {
            const int before = __popcll(same & below);
            const int base = cnt[wave][d];
            rank[i] = base + before;
            if (before == 0) cnt[wave][d] = base + __popcll(same);
        }
    }
    __syncthreads();
    int total = 0;
    if (threadIdx.x < kDigits) {
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const int t = cnt[k][threadIdx.x];
            cnt[k][threadIdx.x] = total;
            total += t;
        }
    }
    const int base = scan_1024(total, wsum);
    if (threadIdx.x < kDigits) {
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) cnt[k][threadIdx.x] += base;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (i >= rounds) continue;
        if ((wave * rounds + i) * 64 + lane < n)
            list[cnt[wave][(key[i] >> (POS_BITS + shift)) & ((1u << bits) - 1u)] + rank[i]] = key[i];
    }
    __syncthreads();
}

// Groups the n keys of list by id (the ids below own): few by comparing each with each, more by digits.
template <int ITEMS, int POS_BITS>
__device__ __forceinline__ void group_ids(uint32_t *list, int n, uint32_t own, int (*cnt)[kDigits], int *wsum)
{
    const int tid = threadIdx.x;
    if (n <= kCompareMax) {               // unique keys: a key's place is the number of smaller ones
        const uint32_t k = tid < n ? list[tid] : 0;
        if (tid >= n && tid < kCompareMax) list[tid] = ~0u;
        __syncthreads();
        int r = 0;
        if (tid < n)
            for (int j = 0; j < n; j += 4) {
                const uint4 x = *reinterpret_cast<const uint4 *>(list + j);
                r += (x.x < k) + (x.y < k) + (x.z < k) + (x.w < k);
            }
        __syncthreads();
        if (tid < n) list[r] = k;
        __syncthreads();
    } else {
        int bits = 1;
        while (((own - 1) >> bits) != 0) ++bits;
        for (int shift = 0; shift < bits; shift += kDigitBits)
            group_list<ITEMS, POS_BITS>(list, n, shift, bits - shift < kDigitBits ? bits - shift : kDigitBits, cnt, wsum);
    }
}

// The whole sort of up to kGroupMax positions in one launch.  Any order of the
// ids serves, as long as equal ids stand together: workgroup g takes the ids
// v = g mod kGroups, looks at every position, keeps those of its ids in
// order, groups them by id, and writes them behind the positions of the
// workgroups before it, which it has counted on the way.  Workgroups past
// kGroups write zeros.  Launches and the trips to memory between them bound
// the sort of so few (16384 positions of 10000 x 100: 14 us, and the call 24.6;
// by digits, four launches, the call 30.0.  4096 of 32000 x 768: 27.1 and 39.2).
__global__ __launch_bounds__(kSortThreads) void group_kernel(const int64_t *__restrict__ ids, int M, uint32_t T, i64 V,
                                                             const float *__restrict__ norm,
                                                             uint32_t *__restrict__ keys, uint32_t *__restrict__ pos,
                                                             int32_t *status, Fill fill)
{
    __shared__ __attribute__((aligned(16))) uint32_t list[kGroupMax];                         // (id / kGroups, position)
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int wsum[kSortWaves], wbelow[kSortWaves], wvalid[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.x >= kGroups) {
        fill_rows(fill, (blockIdx.x - kGroups) * kSortWaves + wave, (gridDim.x - kGroups) * kSortWaves);
        return;
    }
    const uint32_t g = blockIdx.x;
    const uint32_t own = (uint32_t)((V - g + kGroups - 1) / kGroups);
    const int rounds = (M + kSortThreads - 1) / kSortThreads;    // of each wave, on consecutive positions
    const int m0 = wave * rounds * 64 + lane;
    int64_t id[kGroupItems];              // all loads in flight
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i) {
        const int m = m0 + i * 64;
        id[i] = i < rounds && m < M ? ids[m] : 0;
    }
    uint32_t key[kGroupItems];
    int mine_n = 0, below_n = 0, valid_n = 0;
    bool bad = false;
    // the position's sample, by steps of 64 positions
    uint32_t q = (uint32_t)m0 / T, r = (uint32_t)m0 - q * T;
    const uint32_t dq = 64 / T, dr = 64 % T;
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i) {
        key[i] = ~0u;
        if (i >= rounds) continue;
        const int m = m0 + i * 64;
        const bool in = m < M && (norm == nullptr || !(norm[m < M ? q : 0] < 0.0f));
        const uint32_t v = (uint32_t)id[i], its = v % kGroups;
        const bool valid = in && (uint32_t)((uint64_t)id[i] >> 32) == 0 && v < (uint32_t)V;
        bad |= in && !valid;
        const bool mine = valid && its == g;
        if (mine) key[i] = (v / kGroups) << kGroupPosBits | (uint32_t)m;
        mine_n += __popcll(__ballot(mine));
        below_n += __popcll(__ballot(valid && its < g));
        if (g == 0) valid_n += __popcll(__ballot(valid));
        q += dq;
        r += dr;
        if (r >= T) {
            r -= T;
            ++q;
        }
    }
    if (bad && g == 0) raise_flag(status, DP_FLAG_BAD_INDEX);
    if (lane == 0) {
        wsum[wave] = mine_n;
        wbelow[wave] = below_n;
        wvalid[wave] = valid_n;
    }
    __syncthreads();
    int at = 0, n = 0, base = 0, kept = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        at += w < wave ? wsum[w] : 0;
        n += wsum[w];
        base += wbelow[w];
        kept += wvalid[w];
    }
    n = __builtin_amdgcn_readfirstlane(n);
    const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i) {
        const bool mine = key[i] != ~0u;
        const uint64_t in = __ballot(mine);
        if (in == 0) continue;
        if (mine) list[at + __popcll(in & below)] = key[i];
        at += __popcll(in);
    }
    __syncthreads();
    group_ids<kGroupItems, kGroupPosBits>(list, n, own, cnt, wsum);
    for (int e = tid; e < n; e += kSortThreads) {
        const uint32_t k = list[e];
        keys[base + e] = (k >> kGroupPosBits) * kGroups + g;
        pos[base + e] = k & ((1u << kGroupPosBits) - 1u);
    }
    // positions left out stand last
    if (g == 0)
        for (int e = kept + tid; e < M; e += kSortThreads) keys[e] = (uint32_t)V;
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

// Workgroups below walk_blocks add rows; the others write zeros.  STREAM: B and
// the sums pass by the caches (65536 x 2048 of 50000: the call 189 us, 181 so).
template <typename T, int VEC, bool STREAM>
__global__ __launch_bounds__(kWalkThreads) void walk_kernel(
    const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos, const T *__restrict__ B, uint32_t M,
    uint32_t Tn, uint32_t V, i64 D, float scale, const float *__restrict__ norm, float C, uint32_t chunk,
    uint32_t chunks, uint32_t colblocks, uint32_t walk_blocks, float *__restrict__ sum, float *__restrict__ part,
    Fill fill)
{
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= walk_blocks) {
        fill_rows(fill, (blockIdx.x - walk_blocks) * kWalkWaves + wave, (gridDim.x - walk_blocks) * kWalkWaves);
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
        if (!on) return;
        if constexpr (STREAM && VEC >= 4) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) store_stream4(dst + col + i, o.v[i], o.v[i + 1], o.v[i + 2], o.v[i + 3]);
        } else {
            *reinterpret_cast<Out<VEC> *>(dst + col) = o;
        }
    };
    bool open = false;                                       // the last position's id continues in the next chunk
    for (uint32_t q0 = lo; q0 < hi; q0 += 64) {
        // lane l holds sorted position q0 + l: its id, its place, its factor, whether its id ends there
        const uint32_t r = q0 + lane;
        const uint32_t key = r < hi ? keys[r] : V;
        const bool ok = key < V;
        const uint32_t p = ok ? pos[r] : 0;
        const float c = ok && norm != nullptr ? clip_factor(norm[p / Tn], C) : 1.0f;
        const bool ends = ok && (r + 1 >= M || keys[r + 1] != key);
        const uint64_t endm = __ballot(ends);
        const int n = __popcll(__ballot(ok));                // positions left out sort last
        for (int b = 0; b < n; b += kBatch) {
            Row<T, VEC> v[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {               // past the end: position 0's row again, not added
                const uint32_t pj = __builtin_amdgcn_readlane(p, b + j);
                const Row<T, VEC> *row = reinterpret_cast<const Row<T, VEC> *>(Bc + (i64)pj * D);
                if constexpr (STREAM && sizeof(*row) == 16) {
                    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
                    v[j] = __builtin_bit_cast(Row<T, VEC>, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(row)));
                } else {
                    v[j] = *row;
                }
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (b + j >= n) continue;
                const float cj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c), b + j));
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] = fmaf(cj, as_f32(v[j].v[i]), acc[i]);
                open = true;
                if ((endm >> (b + j)) & 1u) {
                    if (here) put(sum + (i64)__builtin_amdgcn_readlane(key, b + j) * D, scale);
                    else put(part + (i64)(2 * ck) * D, 1.0f);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
                    here = true;
                    open = false;
                }
            }
        }
        if (n < 64) break;
    }
    if (open) put(part + (i64)(2 * ck + (here ? 1 : 0)) * D, 1.0f);
}

// Chunk ck's last id, if its positions start in the chunk and continue behind
// it: its piece there, then the following chunks' pieces, added in chunk
// order (each of the four waves a run of them, then the waves in order).
template <int VEC>
__global__ __launch_bounds__(kWalkThreads) void join_kernel(const uint32_t *__restrict__ keys, uint32_t M, uint32_t V,
                                                            i64 D, float scale, uint32_t chunk, uint32_t colblocks,
                                                            float *__restrict__ sum, const float *__restrict__ part,
                                                            uint32_t fill_blocks, Fill fill)
{
    __shared__ float red[kWalkWaves][64 * VEC];
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x < fill_blocks) {       // the zeros first: the pieces' workgroups end sooner
        fill_rows(fill, blockIdx.x * kWalkWaves + wave, fill_blocks * kWalkWaves);
        return;
    }
    const uint32_t unit = blockIdx.x - fill_blocks, ck = unit / colblocks;
    const uint32_t lo = ck * chunk, hi = lo + chunk;         // the grid leaves out the last chunk: hi < M
    const uint32_t key = keys[hi - 1];
    if (key >= V || keys[hi] != key || (lo > 0 && keys[lo - 1] == key)) return;
    // n, the following chunks that hold the id up to their end and behind it: between lo_n and hi_n, 64 places looked
    // at together, first the next 64
    uint32_t n = 0, hi_n = (M - 1) / chunk - (ck + 1), step = 1;
    while (n < hi_n) {
        const uint32_t x = n + (lane + 1) * step;            // chunk ck + x is full
        const uint32_t h = (ck + 1 + x) * chunk;             // its end
        const uint64_t stop = ~__ballot(x <= hi_n && keys[h] == key);
        const uint32_t full = stop != 0 ? __ffsll((unsigned long long)stop) - 1 : 64;
        if (full < 64 && n + (full + 1) * step - 1 < hi_n) hi_n = n + (full + 1) * step - 1;
        n += full * step;
        step = (hi_n - n + 63) / 64;
    }
    ++n;                                                     // and the one in which it ends
    const i64 col = (i64)(unit % colblocks) * 64 * VEC + lane * VEC;
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
    for (uint32_t x = x0; x < x1; x += kBatch) {
        Out<VEC> v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            v[j] = *reinterpret_cast<const Out<VEC> *>(P + (i64)(2 * (x + j < x1 ? x + j : x)) * D);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
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

// ---------------------------------------------------------------------------
// Few positions: one launch.  Workgroup (g, column block) owns the ids
// v = g mod G of its columns.  It looks at every position, keeps those of its
// ids in order, zeroes its rows without a token, groups the kept positions by
// id, and adds the rows: each wave a run of the grouped positions, an id that
// crosses waves joined through LDS in wave order.
// ---------------------------------------------------------------------------
template <typename T, int VEC>
__global__ __launch_bounds__(kSortThreads) void one_kernel(const int64_t *__restrict__ ids, const T *__restrict__ B,
                                                           int M, uint32_t Tn, i64 V, i64 D, float scale,
                                                           const float *__restrict__ norm, float C, int log_g,
                                                           float *__restrict__ sum, int32_t *status)
{
    __shared__ __attribute__((aligned(16))) uint32_t ranked[kOneMax];            // (id / G, position)
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ uint32_t seen[kOneIds / 32];                      // ids of the workgroup that hold a token
    __shared__ Out<VEC> head[kSortWaves][64];                    // pieces of an id that started in an earlier wave
    __shared__ int wsum[kSortWaves];
    __shared__ int passes[kSortWaves];                           // the wave's first id covers its run and goes on
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t G = 1u << log_g, g = blockIdx.x & (G - 1);
    const i64 col = (i64)(blockIdx.x >> log_g) * 64 * VEC + lane * VEC;
    const bool on = col < D;
    const uint32_t own = g < V ? (uint32_t)((V - g + G - 1) >> log_g) : 0;      // ids of the workgroup

    for (uint32_t i = tid; i < (own + 31) / 32; i += kSortThreads) seen[i] = 0;
    bool bad = false;
    uint32_t key[kOneItems];
    int mine_n = 0;
#pragma unroll
    for (int i = 0; i < kOneItems; ++i) {
        const int m = (wave * kOneItems + i) * 64 + lane;
        const int64_t id = m < M ? ids[m] : 0;
        const bool valid = id >= 0 && id < V;
        bool mine = m < M && valid && ((uint32_t)id & (G - 1)) == g;
        // (the norms of few positions are looked at: a division to find the sample, and a load that waits for it)
        if ((mine || !valid) && norm != nullptr && norm[(uint32_t)m / Tn] < 0.0f) mine = false;
        else bad |= !valid;
        key[i] = mine ? (((uint32_t)id >> log_g) << kPosBits) | (uint32_t)m : ~0u;
        mine_n += __popcll(__ballot(mine));
    }
    if (bad && blockIdx.x == 0) raise_flag(status, DP_FLAG_BAD_INDEX);
    if (lane == 0) wsum[wave] = mine_n;
    __syncthreads();
    int at = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        at += w < wave ? wsum[w] : 0;
        n += wsum[w];
    }
    n = __builtin_amdgcn_readfirstlane(n);
    const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
    for (int i = 0; i < kOneItems; ++i) {
        const uint64_t in = __ballot(key[i] != ~0u);
        if (key[i] != ~0u) {
            ranked[at + __popcll(in & below)] = key[i];
            const uint32_t v = key[i] >> kPosBits;
            atomicOr(&seen[v >> 5], 1u << (v & 31));
        }
        at += __popcll(in);
    }
    __syncthreads();
    if (on) {
        Out<VEC> z;
#pragma unroll
        for (int i = 0; i < VEC; ++i) z.v[i] = 0.0f;
        for (uint32_t v = wave; v < own; v += kSortWaves)
            if (((seen[v >> 5] >> (v & 31)) & 1u) == 0)
                *reinterpret_cast<Out<VEC> *>(sum + (((i64)v << log_g) + g) * D + col) = z;
    }
    group_ids<kOneItems, kPosBits>(ranked, n, own, cnt, wsum);

    const int run = (n + kSortWaves - 1) / kSortWaves;
    const int lo = wave * run < n ? wave * run : n, hi = lo + run < n ? lo + run : n;
    const T *Bc = B + (on ? col : 0);
    bool here = lo < hi && (lo == 0 || (ranked[lo - 1] >> kPosBits) != (ranked[lo] >> kPosBits));
    bool open = false;
    uint32_t last = 0;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    const auto take = [&](Out<VEC> &o, float f) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            o.v[i] = f * acc[i];
            acc[i] = 0.0f;
        }
    };
    for (int r0 = lo; r0 < hi; r0 += kBatch) {
        const int r = r0 + (lane & (kBatch - 1));
        const bool ok = r < hi;
        const uint32_t k = ranked[ok ? r : r0];
        const uint32_t p = k & ((1u << kPosBits) - 1u);
        const float c = norm != nullptr ? clip_factor(norm[p / Tn], C) : 1.0f;
        const bool ends = ok && (r + 1 >= n || (ranked[r + 1 < n ? r + 1 : r] >> kPosBits) != (k >> kPosBits));
        const uint32_t endm = (uint32_t)__ballot(ends);
        Row<T, VEC> v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t pj = __builtin_amdgcn_readlane(p, j);
            v[j] = *reinterpret_cast<const Row<T, VEC> *>(Bc + (i64)pj * D);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (r0 + j >= hi) continue;
            const float cj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c), j));
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] = fmaf(cj, as_f32(v[j].v[i]), acc[i]);
            last = __builtin_amdgcn_readlane(k, j) >> kPosBits;
            open = true;
            if ((endm >> j) & 1u) {
                Out<VEC> o;
                take(o, here ? scale : 1.0f);
                if (here) {
                    if (on) *reinterpret_cast<Out<VEC> *>(sum + (((i64)last << log_g) + g) * D + col) = o;
                } else {
                    head[wave][lane] = o;
                }
                here = true;
                open = false;
            }
        }
    }
    const bool through = open && !here;                          // the first id covers the run and goes on
    if (through) take(head[wave][lane], 1.0f);
    if (lane == 0) passes[wave] = through ? 1 : 0;
    __syncthreads();
    if (!open || !here) return;
    // an id that starts in this wave and goes on: the following waves' pieces in wave order
    for (int w = wave + 1; w < kSortWaves; ++w) {
        const Out<VEC> o = head[w][lane];
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += o.v[i];
        if (passes[w] == 0) break;
    }
    if (on) {
        Out<VEC> o;
        take(o, scale);
        *reinterpret_cast<Out<VEC> *>(sum + (((i64)last << log_g) + g) * D + col) = o;
    }
}

// The one-launch path takes up to kOneMax positions: an id's rows are read by
// one workgroup per column block, so that a token on every position costs
// what one CU takes to read them.
bool one_rule(i64 M, i64 V) { return M <= kOneMax && V <= (i64)kOneIds << 12; }

template <typename T>
void one_launch(const int64_t *ids, const void *B, i64 M, i64 T_, i64 V, i64 D, int vec, float scale, const float *norm,
                float C, float *sum, int32_t *status, hipStream_t stream)
{
    const i64 colblocks = ceil_div(D, 64 * (i64)vec);
    // groups of ids: up to 512 workgroups with the column blocks, more where a workgroup would own over kOneIds ids
    int lg = 0;
    while (lg < 9 && (i64(2) << lg) <= V && (colblocks << lg) < 512) ++lg;
    while (((V - 1) >> lg) >= kOneIds) ++lg;
    const unsigned blocks = (unsigned)(colblocks << lg);
    const auto go = [&](auto kernel) {
        kernel<<<blocks, kSortThreads, 0, stream>>>(ids, (const T *)B, (int)M, (uint32_t)T_, V, D, scale, norm, C, lg, sum,
                                                    status);
    };
    if (vec == 8) {
        if constexpr (std::is_same<T, uint16_t>::value) go(one_kernel<T, 8>);
    } else if (vec == 4) {
        go(one_kernel<T, 4>);
    } else if (vec == 2) {
        go(one_kernel<T, 2>);
    } else {
        go(one_kernel<T, 1>);
    }
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

// The groups of rows that each launch zeroes beside its work.  A table of up
// to kFillAllBytes is zeroed whole by the sort's launches, which are bound by
// latency (4096 positions, 32000 x 768: the call 27 us, 35 with the flags;
// 16640, sorted by digits: 50 and 48, where all ids are alike 66 and 80); of
// a larger one only the rows without a token are, once their flags are
// there (65536 positions, 50000 x 2048): up to kFillBytes by each later
// launch that is bound by latency, the rest by the walk.
struct Fills {
    Fill group, count[4], scatter[4], walk, join;
    bool flags;
};

Fills split_fill(const Plan &p, float *sum, char *ws, i64 V, i64 D)
{
    const uint32_t groups = (uint32_t)ceil_div(V, kFillRows);
    Fills f;
    f.flags = 4 * V * D > kFillAllBytes;
    const uint8_t *present = f.flags ? (const uint8_t *)(ws + p.present) : nullptr;
    uint32_t at = 0;
    const auto next = [&](i64 most) {
        const uint32_t n = (uint32_t)(most < groups - at ? most : groups - at);
        const Fill r = {sum, present, (uint32_t)V, at, at + n, D};
        at += n;
        return r;
    };
    const i64 part = f.flags ? kFillBytes / (4 * D * kFillRows) + 1 : ceil_div(groups, 2 * p.passes);
    f.group = next(p.grouped ? groups : 0);
    for (int i = 0; i < p.passes; ++i) {
        f.count[i] = next(f.flags && i == 0 ? 0 : part);
        f.scatter[i] = next(f.flags && i == 0 ? 0 : part);
    }
    f.join = next(p.chunks > 1 ? part : 0);
    f.walk = next(groups);
    return f;
}

// workgroups of `waves` waves for a fill
uint32_t fill_blocks(const Fill &f, int waves)
{
    const i64 b = ceil_div(f.g1 - f.g0, waves);
    return (uint32_t)(b < kFillBlocks ? b : kFillBlocks);
}

template <typename T, int VEC>
void sums(const Plan &p, const void *B, i64 T_, i64 V, i64 D, float scale, const float *norm, float C, float *sum,
          char *ws, int buf, const Fills &fills, hipStream_t stream)
{
    const uint32_t *keys = (const uint32_t *)(ws + p.keys[buf]), *pos = (const uint32_t *)(ws + p.pos[buf]);
    float *part = (float *)(ws + p.part);
    const uint32_t walk_blocks = (uint32_t)ceil_div(p.chunks * p.colblocks, kWalkWaves);
    const uint32_t blocks = walk_blocks + fill_blocks(fills.walk, kWalkWaves);
    const auto walk = [&](auto kernel) {
        kernel<<<blocks, kWalkThreads, 0, stream>>>(keys, pos, (const T *)B, (uint32_t)p.M, (uint32_t)T_, (uint32_t)V, D,
                                                    scale, norm, C, (uint32_t)p.chunk, (uint32_t)p.chunks,
                                                    (uint32_t)p.colblocks, walk_blocks, sum, part, fills.walk);
    };
    constexpr bool WIDE = sizeof(T) * VEC == 16;
    if (WIDE && fills.flags) walk(walk_kernel<T, VEC, WIDE>);
    else walk(walk_kernel<T, VEC, false>);
    if (p.chunks > 1) {
        const uint32_t fb = fill_blocks(fills.join, kWalkWaves);
        join_kernel<VEC><<<(unsigned)((p.chunks - 1) * p.colblocks) + fb, kWalkThreads, 0, stream>>>(
            keys, (uint32_t)p.M, (uint32_t)V, D, scale, (uint32_t)p.chunk, (uint32_t)p.colblocks, sum, part, fb,
            fills.join);
    }
}

template <typename T>
void sums_by_vec(const Plan &p, const void *B, i64 T_, i64 V, i64 D, float scale, const float *norm, float C,
                 float *sum, char *ws, int buf, const Fills &fills, hipStream_t stream)
{
    if (p.vec == 8) {
        if constexpr (std::is_same<T, uint16_t>::value)
            sums<T, 8>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, fills, stream);
    } else if (p.vec == 4) {
        sums<T, 4>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, fills, stream);
    } else if (p.vec == 2) {
        sums<T, 2>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, fills, stream);
    } else {
        sums<T, 1>(p, B, T_, V, D, scale, norm, C, sum, ws, buf, fills, stream);
    }
}

// Sorts the positions; returns which of the two buffers holds the result.
template <int ITEMS>
int sort(const Plan &p, const int64_t *ids, i64 T, i64 V, const float *norm, int32_t *status, char *ws,
         const Fills &fills, hipStream_t stream)
{
    int32_t *hist = (int32_t *)(ws + p.hist);
    int32_t *tot = p.tiles > kScanTiles ? (int32_t *)(ws + p.tot) : nullptr;
    uint8_t *present = fills.flags ? (uint8_t *)(ws + p.present) : nullptr;
    const unsigned tiles = (unsigned)p.tiles;
    int buf = 0;
    for (int i = 0; i < p.passes; ++i, buf ^= 1) {
        uint32_t *ki = (uint32_t *)(ws + p.keys[buf]), *ko = (uint32_t *)(ws + p.keys[buf ^ 1]);
        uint32_t *pi = (uint32_t *)(ws + p.pos[buf]), *po = (uint32_t *)(ws + p.pos[buf ^ 1]);
        const Fill &fc = fills.count[i], &fs = fills.scatter[i];
        if (i == 0)
            count_kernel<ITEMS, true><<<tiles + fill_blocks(fc, kSortWaves), kSortThreads, 0, stream>>>(
                ids, (uint32_t)p.M, (uint32_t)T, V, norm, ki, 0, p.bits, hist, (int)tiles, p.hist_ld, present, status, fc);
        else
            count_kernel<ITEMS, false><<<tiles + fill_blocks(fc, kSortWaves), kSortThreads, 0, stream>>>(
                ids, (uint32_t)p.M, (uint32_t)T, V, norm, ki, i * p.bits, p.bits, hist, (int)tiles, p.hist_ld, present,
                status, fc);
        if (tot != nullptr) scan_kernel<<<1u << p.bits, kSortThreads, 0, stream>>>(hist, tot, (int)p.tiles);
        scatter_kernel<ITEMS><<<tiles + fill_blocks(fs, kSortWaves), kSortThreads, 0, stream>>>(
            ki, i == 0 ? nullptr : pi, ko, po, (uint32_t)p.M, V, i * p.bits, p.bits, hist, tot, (int)tiles, p.hist_ld,
            present, fs);
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
    // a grid holds fewer than 2^24 workgroups of 256: one per 256 positions and 64 columns at the most, or (one_kernel)
    // 2^22 of 1024: one per 8192 ids and 64 columns
    DPG_REQUIRE(N * T * D < (i64(1) << 37) && V * D < (i64(1) << 38), DP_EUNSUPPORTED);
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
    const int vec = vec_for(B, sum, dt, D);
    if (one_rule(N * T, V)) {
        if (dt == DP_F32) one_launch<float>(ids, B, N * T, T, V, D, vec, scale, norm, C, sum, status, stream);
        else one_launch<uint16_t>(ids, B, N * T, T, V, D, vec, scale, norm, C, sum, status, stream);
        return launch_status();
    }
    const Plan p = make_plan(N, T, V, D, vec);
    char *w = (char *)ws;
    const Fills fills = split_fill(p, sum, w, V, D);
    int buf = 0;
    if (p.grouped)
        group_kernel<<<kGroups + fill_blocks(fills.group, kSortWaves), kSortThreads, 0, stream>>>(
            ids, (int)p.M, (uint32_t)T, V, norm, (uint32_t *)(w + p.keys[0]), (uint32_t *)(w + p.pos[0]),
            status, fills.group);
    else
        buf = p.items == 2 ? sort<2>(p, ids, T, V, norm, status, w, fills, stream)
                           : sort<8>(p, ids, T, V, norm, status, w, fills, stream);
    if (dt == DP_F32) sums_by_vec<float>(p, B, T, V, D, scale, norm, C, sum, w, buf, fills, stream);
    else sums_by_vec<uint16_t>(p, B, T, V, D, scale, norm, C, sum, w, buf, fills, stream);
    return launch_status();
}
