// Blocks of rows and of keys in the order of their work, the longest first.
//
// With documents packed in samples a block's work follows from where its
// documents end, which only the device knows; in the order of positions a long
// block may start last and leave the card waiting for it (two samples of 8192 in
// four documents of 1 : 2 : 3 : 4, 16 key heads: dK and dV's 64 blocks a head
// took 1717 us so, and 1260 in this order; the ranking itself takes 31).  One workgroup per order counts the tiles of 64 that each
// block meets, by their documents' ranges as the kernels do, and ranks the
// blocks by comparing all pairs.  The order decides when a block runs, not what
// it computes.
#include "attention_order.hpp"

#include "attention_tile.hpp"

namespace dpg {
namespace attn {
namespace {

constexpr int kThreads = 1024, kTile = 64, kBlock = 128;
constexpr int kMaxTiles = 4096, kMaxEntries = 2048;

__global__ __launch_bounds__(kThreads) void order_kernel(Call c, int32_t *rows, int32_t *keys)
{
    __shared__ int lo[kMaxTiles], hi[kMaxTiles], work[kMaxEntries];
    const bool of_rows = blockIdx.x == 0 && rows != nullptr;
    int32_t *order = of_rows ? rows : keys;
    const int M = c.Tq * c.G, tiles = (c.Tk + kTile - 1) / kTile;
    const int blocks = of_rows ? (M + kBlock - 1) / kBlock : (c.Tk + kBlock - 1) / kBlock, entries = c.N * blocks;
    for (int e = threadIdx.x; e < c.N * tiles; e += kThreads) {
        const Sample s(c, e / tiles);
        const int p0 = e % tiles * kTile, p1 = p0 + kTile < s.L ? p0 + kTile : s.L;
        docs_range(s.docs, p0, p1, lo[e], hi[e]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < entries; e += kThreads) {
        const int n = e / blocks, b = e - n * blocks;
        const Sample s(c, n);
        const int *l = lo + n * tiles, *h = hi + n * tiles;
        // the block's positions, and the tiles that may meet it
        int p0, p1, t0 = 0, t1;
        if (of_rows) {
            const RowSpan r = span_of(s, c.G, M, b * kBlock, kBlock);
            p0 = r.pmin;
            p1 = r.pmax + 1;
            t1 = p1 > p0 ? (s.end_for(r.pmax) + kTile - 1) / kTile : 0;
        } else {
            p0 = b * kBlock;
            p1 = p0 + kBlock < s.L ? p0 + kBlock : s.L;
            const int queries = s.L < c.Tq ? s.L : c.Tq;
            if (s.causal && p0 >= s.prefix) t0 = p0 / kTile;
            t1 = p1 > p0 ? (queries + kTile - 1) / kTile : 0;
        }
        int d0 = 0x7fffffff, d1 = -0x7fffffff - 1, count = 0;
        for (int t = p0 / kTile; t * kTile < p1; ++t) {
            d0 = l[t] < d0 ? l[t] : d0;
            d1 = h[t] > d1 ? h[t] : d1;
        }
        for (int t = t0; t < t1; ++t) count += l[t] <= d1 && h[t] >= d0 && h[t] >= 0 ? 1 : 0;
        work[e] = count;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < entries; e += kThreads) {
        const int w = work[e];
        int rank = 0;
#pragma unroll 8
        for (int o = 0; o < entries; ++o) rank += work[o] > w || (work[o] == w && o < e) ? 1 : 0;
        order[rank] = e;
    }
}

i64 entries_of(const dp_attention &a, i64 blocks)
{
    if (a.docs == nullptr || (a.flags & DP_ATTENTION_LAST) != 0 || a.Tk < 1024) return 0;
    if (a.N * ceil_div(a.Tk, kTile) > kMaxTiles || a.N * blocks > kMaxEntries) return 0;
    return a.N * a.Hk * blocks >= 256 ? a.N * blocks : 0;
}

}  // namespace

i64 row_order_entries(const dp_attention &a) { return entries_of(a, ceil_div(a.Tq * (a.Hq / a.Hk), kBlock)); }
i64 key_order_entries(const dp_attention &a) { return entries_of(a, ceil_div(a.Tk, kBlock)); }

void order_blocks(const Call &c, int32_t *rows, int32_t *keys, hipStream_t stream)
{
    if (rows == nullptr && keys == nullptr) return;
    order_kernel<<<rows != nullptr && keys != nullptr ? 2 : 1, kThreads, 0, stream>>>(c, rows, keys);
}

}  // namespace attn
}  // namespace dpg
