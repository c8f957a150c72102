// Embedding forward: Y[m][:] = s * E[ids[m]][:].
//
// Nothing is computed but one product per element, so the call is bound by
// its bytes: each looked-up row once (repeated ids come from the caches) and
// the output once.  A group of L lanes (L a power of two, as few as cover a
// row in one sweep) takes one row: one id load, then all of the group's
// kSweeps loads in flight, then its stores.  A row longer than kSweeps sweeps
// is split over blockIdx.y, so that a single token still has all its loads in
// flight at once.  Outputs of more than kStreamBytes are stored past the caches,
// which then hold more of the table (65536 rows of 4096, fp32 to bf16, 537 MB
// written and 310 MB of distinct rows read: 184 us, 172 so, 4.9 TB/s).
#include "common.hpp"

namespace dpg {
namespace {

constexpr int kThreads = 256;
constexpr int kSweeps = 4;
constexpr i64 kMaxGrid = i64(1) << 22;
constexpr i64 kStreamBytes = i64(96) << 20;

__device__ __forceinline__ uint16_t f32_to_bf16(float x)
{
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}

// VEC consecutive elements, as loaded: 16-byte pieces where VEC elements hold that many bytes
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC < 16 ? sizeof(T) * VEC : 16) Pack {
    T v[VEC];
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ void from_f32(float x, float &y) { y = x; }
__device__ __forceinline__ void from_f32(float x, uint16_t &y) { y = f32_to_bf16(x); }

template <typename TE, typename TY, int VEC, bool STREAM>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const int64_t *__restrict__ ids, const TE *__restrict__ E,
                                                          i64 M, i64 V, int D, int log_l, float scale,
                                                          TY *__restrict__ Y, int32_t *status)
{
    const int L = 1 << log_l;
    const int sub = threadIdx.x & (L - 1);
    const int rows = kThreads >> log_l;
    const int d0 = (int)blockIdx.y * (kSweeps * VEC << log_l) + sub * VEC;
    for (i64 m = (i64)blockIdx.x * rows + (threadIdx.x >> log_l); m < M; m += (i64)gridDim.x * rows) {
        const int64_t id = ids[m];
        const bool ok = id >= 0 && id < V;
        if (!ok && sub == 0 && blockIdx.y == 0) raise_flag(status, DP_FLAG_BAD_INDEX);
        const TE *e = E + (ok ? id : 0) * (i64)D;
        TY *y = Y + m * (i64)D;
        Pack<TE, VEC> in[kSweeps];
#pragma unroll
        for (int k = 0; k < kSweeps; ++k) {
            const int d = d0 + (k * VEC << log_l);
            // past the end: the row's first elements again, not stored
            in[k] = *reinterpret_cast<const Pack<TE, VEC> *>(e + (d < D ? d : 0));
        }
#pragma unroll
        for (int k = 0; k < kSweeps; ++k) {
            const int d = d0 + (k * VEC << log_l);
            if (d < D) {
                Pack<TY, VEC> out;
#pragma unroll
                for (int i = 0; i < VEC; ++i) from_f32(ok ? scale * to_f32(in[k].v[i]) : 0.0f, out.v[i]);
                if constexpr (STREAM) {           // pieces of at most 16 bytes, as the rows are aligned
                    constexpr int W = sizeof(out) < 16 ? sizeof(out) / 4 : 4, PIECES = sizeof(out) / (4 * W);
                    typedef uint32_t piece_t __attribute__((ext_vector_type(W)));
                    struct Pieces {
                        piece_t v[PIECES];
                    };
                    const Pieces p = __builtin_bit_cast(Pieces, out);
#pragma unroll
                    for (int i = 0; i < PIECES; ++i)
                        __builtin_nontemporal_store(p.v[i], reinterpret_cast<piece_t *>(y + d) + i);
                } else {
                    *reinterpret_cast<Pack<TY, VEC> *>(y + d) = out;
                }
            }
        }
    }
}

template <typename TE, typename TY, int VEC>
dp_status launch(const int64_t *ids, const void *E, i64 M, i64 V, i64 D, float scale, void *Y, int32_t *status,
                 hipStream_t stream)
{
    int log_l = 0;
    while (log_l < 6 && (i64)(VEC << log_l) < D) ++log_l;
    const i64 rows = kThreads >> log_l, cols = (i64)kSweeps * VEC << log_l;
    // a dimension of a grid holds fewer than 2^32 threads: past kMaxGrid workgroups each takes several rounds of rows
    const i64 gx = ceil_div(M, rows);
    const dim3 grid((unsigned)(gx < kMaxGrid ? gx : kMaxGrid), (unsigned)ceil_div(D, cols));
    const bool past = VEC >= 4 && sizeof(TY) * M * D > kStreamBytes;
    const auto go = [&](auto kernel) {
        kernel<<<grid, kThreads, 0, stream>>>(ids, (const TE *)E, M, V, (int)D, log_l, scale, (TY *)Y, status);
    };
    if (past) go(lookup_kernel<TE, TY, VEC, (VEC >= 4)>);
    else go(lookup_kernel<TE, TY, VEC, false>);
    return launch_status();
}

template <typename TE, typename TY>
dp_status by_vec(const int64_t *ids, const void *E, i64 M, i64 V, i64 D, float scale, void *Y, int32_t *status,
                 hipStream_t stream)
{
    // the widest loads and stores that every row start allows
    const auto fits = [&](int vec) {
        const size_t be = sizeof(TE) * vec < 16 ? sizeof(TE) * vec : 16, by = sizeof(TY) * vec < 16 ? sizeof(TY) * vec : 16;
        return D % vec == 0 && aligned(E, be) && aligned(Y, by);
    };
    if (fits(8)) return launch<TE, TY, 8>(ids, E, M, V, D, scale, Y, status, stream);
    if (fits(4)) return launch<TE, TY, 4>(ids, E, M, V, D, scale, Y, status, stream);
    return launch<TE, TY, 1>(ids, E, M, V, D, scale, Y, status, stream);
}

}  // namespace
}  // namespace dpg

using namespace dpg;

extern "C" dp_status dp_embedding_lookup(const int64_t *ids, const void *E, dp_dtype dt, int64_t N, int64_t T,
                                         int64_t V, int64_t D, float scale, void *Y, dp_dtype dt_y, int32_t *status,
                                         hipStream_t stream)
{
    DPG_REQUIRE(dtype_ok(dt) && dtype_ok(dt_y), DP_EDTYPE);
    DPG_REQUIRE(N >= 0 && T >= 0 && V >= 1 && D >= 1, DP_EINVAL);
    DPG_REQUIRE(V < (i64(1) << 31), DP_EINVAL);
    DPG_REQUIRE(N < (i64(1) << 31) && T < (i64(1) << 31) && N * T < (i64(1) << 31), DP_EUNSUPPORTED);
    DPG_REQUIRE(D < (i64(1) << 23), DP_EUNSUPPORTED);       // blockIdx.y counts 256-column pieces
    const i64 M = N * T;
    if (M == 0) return DP_OK;
    DPG_REQUIRE(ids != nullptr && E != nullptr && Y != nullptr, DP_EINVAL);
    if (dt == DP_F32)
        return dt_y == DP_F32 ? by_vec<float, float>(ids, E, M, V, D, scale, Y, status, stream)
                              : by_vec<float, uint16_t>(ids, E, M, V, D, scale, Y, status, stream);
    return dt_y == DP_F32 ? by_vec<uint16_t, float>(ids, E, M, V, D, scale, Y, status, stream)
                          : by_vec<uint16_t, uint16_t>(ids, E, M, V, D, scale, Y, status, stream);
}
