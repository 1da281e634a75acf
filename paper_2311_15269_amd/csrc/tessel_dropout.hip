// Dropout whose mask is never stored (formulas: include/tessel_block_ops.h): one pass, eight channels a lane.
//
// Bound by memory: 8192 x 4096 bf16 in 21.2 us (134 MB, 6.3 TB/s), 26.6 where every call is on other memory than the last (5.0 TB/s, a large copy's rate); 4999 x 1003 in 32 bits
// in 7.7 (5.2 TB/s, 2.3 of them the launch and the first reads).  Philox's two counters for eight values are 64 instructions behind what their columns share, half of the time
// that memory leaves; rows of few channels, of which a counter of four words serves one to four values, are bound by it (2^24 x 1 in 57 us, 1.2 TB/s).
#include "tessel_draw.h"

namespace tessel {

constexpr int kThreads = 256;

template <typename T, bool WIDE, int ROWS>
__global__ __launch_bounds__(kThreads) void dropout_kernel(tessel_dropout_rows a, DropLaunch l, int lanes)
{
    const Span<WIDE, ROWS> at(a.channels, lanes);
    typename Eight<T>::type x[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; r++) x[r] = read8<T, !WIDE>((const T *)a.x.data + min(at.token + r * at.step, a.tokens - 1) * a.x.stride, at.col, a.channels);
    const Draw draw(l, a.channels, at.col);
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        const int64_t token = at.token + r * at.step;
        if (token >= a.tokens) break;
        float v[8];
        place8<T, !WIDE>(at.col, a.channels, x[r]);
        widen8<T>(v, x[r]);
        if (l.least) draw.apply(v, (uint32_t)token);
        store8<T>((T *)a.y.data + token * a.y.stride, v, at.col, a.channels);
    }
}

int launch_dropout(const tessel_dropout_rows &a, const DropLaunch &d, void *stream)
{
    tessel_dropout_rows aa = a;
    DropLaunch dd = d;
    const int rows = span_rows(a.type, a.tokens, a.channels, d, 256);
    SpanShape s = span_shape(a.tokens, a.channels, rows);
    void *args[] = {&aa, &dd, &s.lanes};
#define KERNEL(T) (s.wide ? rows == 4 ? (const void *)dropout_kernel<T, true, 4> : (const void *)dropout_kernel<T, true, 1> \
                          : rows == 4 ? (const void *)dropout_kernel<T, false, 4> : (const void *)dropout_kernel<T, false, 1>)
    return launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)s.groups), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

}  // namespace tessel
