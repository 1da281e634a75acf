// Dropout whose mask is never stored (formulas: include/tessel_block_ops.h): eight channels a lane, two words' counters each.
#include "tessel_draw.h"

namespace tessel {

constexpr int kThreads = 256;

template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(tessel_dropout_rows a, DropLaunch d)
{
    const uint32_t per = (uint32_t)(((int64_t)a.channels + 7) / 8);
    const uint64_t n = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const uint32_t row = (uint32_t)(n / per);
    const int col = (int)(n % per) * 8;
    if ((int64_t)(n / per) >= a.tokens) return;
    float v[8];
    load8<T>(v, (const T *)a.x.data + row * a.x.stride, col, a.channels);
    if (d.least) drop8(v, d, number_of(d), row, col);
    store8<T>((T *)a.y.data + row * a.y.stride, v, col, a.channels);
}

int launch_dropout(const tessel_dropout_rows &a, const DropLaunch &d, void *stream)
{
    tessel_dropout_rows aa = a;
    DropLaunch dd = d;
    void *args[] = {&aa, &dd};
    const int64_t lanes = a.tokens * (((int64_t)a.channels + 7) / 8);
#define KERNEL(T) ((const void *)dropout_kernel<T>)
    return launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)((lanes + kThreads - 1) / kThreads)), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

}  // namespace tessel
