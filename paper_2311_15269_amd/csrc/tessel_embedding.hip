// The embedding of a shard of the vocabulary, forward and backward (formulas: include/tessel_block_ops.h).
//
// Forward: eight channels of a token a lane.  Backward: a workgroup for every row of the table looks through all tokens for its own, in order.
#include "tessel_draw.h"

namespace tessel {

constexpr int kThreads = 256;

// the row of the table that token t takes, -1 if there is none
__device__ __forceinline__ int row_at(const tessel_embedding &a, int64_t t)
{
    const int64_t v = a.index_type == TESSEL_I64 ? ((const int64_t *)a.token)[t] : ((const int32_t *)a.token)[t];
    return v >= a.first && v - a.first < a.rows ? (int)(v - a.first) : -1;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void embed_kernel(tessel_embedding a, DropLaunch d)
{
    const uint32_t per = (uint32_t)(((int64_t)a.channels + 7) / 8);
    const uint64_t n = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = (int64_t)(n / per);
    const int col = (int)(n % per) * 8;
    if (t >= a.tokens) return;
    const int row = row_at(a, t);
    float v[8] = {};
    if (row >= 0) {
        load8<T>(v, (const T *)a.table.data + row * a.table.stride, col, a.channels);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] *= a.scale;
        if (d.least) drop8(v, d, number_of(d), (uint32_t)t, col);
    }
    store8<T>((T *)a.out.data + t * a.out.stride, v, col, a.channels);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void embed_backward_kernel(tessel_embedding a, DropLaunch d)
{
    __shared__ uint64_t found[kThreads / 64];
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int first = 0; first < a.channels; first += 8 * kThreads) {
        const int col = first + 8 * threadIdx.x;
        float sum[8] = {};
        bool any = false;
        for (int64_t t0 = 0; t0 < a.tokens; t0 += kThreads) {
            const bool mine = t0 + threadIdx.x < a.tokens && row_at(a, t0 + threadIdx.x) == row;
            const uint64_t mask = __ballot(mine);
            if (lane == 0) found[wave] = mask;
            __syncthreads();
            for (int w = 0; w < kThreads / 64; w++)
                for (uint64_t m = found[w]; m; m &= m - 1) {
                    const int64_t t = t0 + 64 * w + __builtin_ctzll(m);
                    float v[8];
                    load8<T>(v, (const T *)a.d_out.data + t * a.d_out.stride, col, a.channels);
                    if (d.least) drop8(v, d, number_of(d), (uint32_t)t, col);
#pragma unroll
                    for (int j = 0; j < 8; j++) sum[j] += v[j];
                    any = true;
                }
            __syncthreads();
        }
        float *to = a.dtable + row * a.dtable_stride;
        if (a.accumulate) {
            if (!any) continue;
            float v[8];
            load8<float>(v, to, col, a.channels);
#pragma unroll
            for (int j = 0; j < 8; j++) sum[j] = v[j] + a.scale * sum[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) sum[j] *= a.scale;
        }
        store8<float>(to, sum, col, a.channels);
    }
}

int launch_embed(const tessel_embedding &a, const DropLaunch &d, void *stream)
{
    tessel_embedding aa = a;
    DropLaunch dd = d;
    void *args[] = {&aa, &dd};
    const int64_t lanes = a.tokens * (((int64_t)a.channels + 7) / 8);
#define KERNEL(T) ((const void *)embed_kernel<T>)
    return launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)((lanes + kThreads - 1) / kThreads)), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

size_t embed_workspace(const tessel_embedding &) { return 0; }

int launch_embed_backward(const tessel_embedding &a, const DropLaunch &d, void *, void *stream)
{
    tessel_embedding aa = a;
    DropLaunch dd = d;
    void *args[] = {&aa, &dd};
#define KERNEL(T) ((const void *)embed_backward_kernel<T>)
    return launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)a.rows), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

}  // namespace tessel
