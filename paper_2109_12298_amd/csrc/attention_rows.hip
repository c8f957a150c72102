// Attention by rows (attention_rows.hpp), for heads wider than the tiles hold.
#include "attention_rows.hpp"

namespace dpg {
namespace attn {
namespace {

constexpr int kThreads = 256, kRows = kThreads / kWave;

// rows in the order [N][H][T]
template <typename T>
__global__ __launch_bounds__(kThreads) void rows_forward_kernel(Call c, T *O, float *lse)
{
    for (i64 r = (i64)blockIdx.x * kRows + threadIdx.x / kWave; r < (i64)c.N * c.Hq * c.Tq; r += (i64)gridDim.x * kRows) {
        const i64 nh = r / c.Tq;
        forward_row<T>(c, (int)(nh / c.Hq), (int)(nh % c.Hq), (int)(r % c.Tq), O, lse);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rows_backward_query_kernel(Call c, const T *O, const float *lse, const T *dO, T *dQ,
                                                                       float *row_delta)
{
    for (i64 r = (i64)blockIdx.x * kRows + threadIdx.x / kWave; r < (i64)c.N * c.Hq * c.Tq; r += (i64)gridDim.x * kRows) {
        const i64 nh = r / c.Tq;
        backward_query_row<T>(c, (int)(nh / c.Hq), (int)(nh % c.Hq), (int)(r % c.Tq), O, lse, dO, dQ, row_delta + r);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rows_backward_key_kernel(Call c, const float *lse, const float *row_delta,
                                                                     const T *dO, T *dK, T *dV)
{
    for (i64 r = (i64)blockIdx.x * kRows + threadIdx.x / kWave; r < (i64)c.N * c.Hk * c.Tk; r += (i64)gridDim.x * kRows) {
        const i64 nh = r / c.Tk;
        backward_key_row<T>(c, (int)(nh / c.Hk), (int)(nh % c.Hk), (int)(r % c.Tk), lse, row_delta, c.Tq, dO, dK, dV);
    }
}

// a dimension of a grid holds fewer than 2^32 threads: past kMaxGrid workgroups a wave takes several rows
constexpr i64 kMaxGrid = i64(1) << 22;
unsigned blocks(i64 rows) { return (unsigned)(ceil_div(rows, kRows) < kMaxGrid ? ceil_div(rows, kRows) : kMaxGrid); }

template <typename T>
dp_status backward(const Call &c, const void *O, const float *lse, const void *dO, void *dQ, void *dK, void *dV,
                   float *row_delta, hipStream_t stream)
{
    const i64 q = (i64)c.N * c.Hq * c.Tq, k = (i64)c.N * c.Hk * c.Tk;
    if (q > 0)
        rows_backward_query_kernel<T><<<blocks(q), kThreads, 0, stream>>>(c, (const T *)O, lse, (const T *)dO, (T *)dQ, row_delta);
    if (k > 0)
        rows_backward_key_kernel<T><<<blocks(k), kThreads, 0, stream>>>(c, lse, row_delta, (const T *)dO, (T *)dK, (T *)dV);
    return launch_status();
}

}  // namespace

dp_status rows_forward(const Call &c, dp_dtype dt, void *O, float *lse, hipStream_t stream)
{
    const i64 q = (i64)c.N * c.Hq * c.Tq;
    if (dt == DP_F32) rows_forward_kernel<float><<<blocks(q), kThreads, 0, stream>>>(c, (float *)O, lse);
    else rows_forward_kernel<uint16_t><<<blocks(q), kThreads, 0, stream>>>(c, (uint16_t *)O, lse);
    return launch_status();
}

dp_status rows_backward(const Call &c, dp_dtype dt, const void *O, const float *lse, const void *dO, void *dQ, void *dK,
                        void *dV, void *ws, hipStream_t stream)
{
    return dt == DP_F32 ? backward<float>(c, O, lse, dO, dQ, dK, dV, (float *)ws, stream)
                        : backward<uint16_t>(c, O, lse, dO, dQ, dK, dV, (float *)ws, stream);
}

}  // namespace attn
}  // namespace dpg
