// Activation checkpoints in 8 bits: store, restore, and the gated activation with its backward pass from them (formulas:
// include/tessel_block_ops.h).  One pass over the data, eight channels a lane, a group of 64 in eight lanes, whose largest value three
// exchanges between lanes find.  Bound by memory: 8192 rows of 4096 bf16 to 8 bits in 21 us (4.9 TB/s), back in 16; 8192 rows of 16384,
// gated: 202 us forward with both checkpoints (5.3 TB/s), 184 back from them.
#include "tessel_rows.h"

namespace tessel {

constexpr int kThreads = 256;

// A lane's place: chunk of eight channels `col / 8` of row `row`.  Rows are counted in whole groups, so that the eight lanes of a group
// are neighbours and either all of them have a row or none has.
struct Place {
    uint32_t row, col;
};
__device__ __forceinline__ bool place_of(int64_t tokens, int channels, Place &p)
{
    const uint32_t per = (uint32_t)((channels + kGroup - 1) / kGroup) * 8u;
    const uint32_t n = blockIdx.x * kThreads + threadIdx.x;      // (the host sees to it that this does not pass 32 bits)
    p.row = n / per;
    p.col = n % per * 8u;
    return p.row < tokens;
}

__device__ __forceinline__ void put_held(const tessel_checkpoint &c, const Place &p, uint2 bytes, uint32_t e)
{
    *(uint2 *)(c.values + p.row * c.value_stride + p.col) = bytes;          // (value_stride: whole groups)
    if (p.col % kGroup == 0) c.exponents[p.row * c.exponent_stride + p.col / kGroup] = (uint8_t)e;
}

__device__ __forceinline__ void get_held(const tessel_checkpoint &c, const Place &p, float *v)
{
    const uint2 bytes = *(const uint2 *)(c.values + p.row * c.value_stride + p.col);
    held8(v, bytes, c.exponents[p.row * c.exponent_stride + p.col / kGroup]);
}

template <typename T>
__device__ __forceinline__ T *row_of(const tessel_rows &r, uint32_t row) { return (T *)r.data + row * r.stride; }

template <typename T>
__global__ __launch_bounds__(kThreads) void store_kernel(tessel_checkpoint c, tessel_rows x)
{
    Place p;
    if (!place_of(c.tokens, c.channels, p)) return;
    float v[8];
    load8<T>(v, row_of<T>(x, p.row), p.col, c.channels);
    uint2 bytes;
    const uint32_t e = hold8<T>(v, bytes);
    put_held(c, p, bytes, e);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void restore_kernel(tessel_checkpoint c, tessel_rows x)
{
    Place p;
    if (!place_of(c.tokens, c.channels, p)) return;
    float v[8];
    get_held(c, p, v);
    store8<T>(row_of<T>(x, p.row), v, p.col, c.channels);
}

// 1 / (1 + exp(-z)): for 16-bit results by the instructions for powers of two and reciprocals, whose error (2^-21 at |z| = 10) is far below theirs
template <typename T>
__device__ __forceinline__ float logistic(float z)
{
    if constexpr (__is_same(T, float)) return 1.0f / (1.0f + expf(-z));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

// an activation and its derivative
template <typename T, int ACT>
__device__ __forceinline__ float activation(float z, float &slope)
{
    if constexpr (ACT == TESSEL_SILU) {
        const float s = logistic<T>(z);
        slope = s * (1.0f + z * (1.0f - s));
        return z * s;
    } else {
        const float root = 0.7978845608028654f, cube = 0.044715f;
        // tanh(w) = 1 - 2 / (1 + exp(2 w)); half of 1 + tanh is s = 1 / (1 + exp(-2 w))
        const float s = logistic<T>(2.0f * root * (z + cube * z * z * z));
        // (s (1 - s) is nought long before the square leaves 32 bits, and z s is z at most, where 2 z may be infinite)
        slope = s + z * s * (1.0f - s) * (2.0f * root) * (1.0f + 3.0f * cube * fminf(z * z, 1e6f));
        return z * s;
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void gated_kernel(tessel_rows g, tessel_rows u, tessel_rows a, tessel_checkpoint kg, tessel_checkpoint ku)
{
    Place p;
    if (!place_of(kg.tokens, kg.channels, p)) return;
    float x[8], y[8], z[8], slope;
    load8<T>(x, row_of<T>(g, p.row), p.col, kg.channels);
    load8<T>(y, row_of<T>(u, p.row), p.col, kg.channels);
    uint2 bytes;
    uint32_t e = hold8<T>(x, bytes);
    put_held(kg, p, bytes, e);
    e = hold8<T>(y, bytes);
    put_held(ku, p, bytes, e);
#pragma unroll
    for (int j = 0; j < 8; j++) z[j] = activation<T, ACT>(x[j], slope) * y[j];
    store8<T>(row_of<T>(a, p.row), z, p.col, kg.channels);
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void gated_backward_kernel(tessel_rows da, tessel_checkpoint kg, tessel_checkpoint ku, tessel_rows dg,
                                                                 tessel_rows du, tessel_rows a)
{
    Place p;
    if (!place_of(kg.tokens, kg.channels, p)) return;
    float x[8], y[8], d[8], z[8];
    load8<T>(d, row_of<T>(da, p.row), p.col, kg.channels);
    get_held(kg, p, x);
    get_held(ku, p, y);
#pragma unroll
    for (int j = 0; j < 8; j++) {
        float slope;
        const float f = activation<T, ACT>(x[j], slope);
        z[j] = f * y[j];
        x[j] = d[j] * y[j] * slope;
        y[j] = d[j] * f;
    }
    store8<T>(row_of<T>(dg, p.row), x, p.col, kg.channels);
    store8<T>(row_of<T>(du, p.row), y, p.col, kg.channels);
    if (a.data) store8<T>(row_of<T>(a, p.row), z, p.col, kg.channels);
}

static dim3 grid_of(const tessel_checkpoint &c)
{
    const uint64_t lanes = (uint64_t)c.tokens * (uint64_t)((c.channels + kGroup - 1) / kGroup) * 8u;
    return dim3((unsigned)((lanes + kThreads - 1) / kThreads));
}

#define BY_TYPE(type, call) ((type) == TESSEL_BF16 ? call(bf16) : (type) == TESSEL_F16 ? call(f16) : call(float))

int launch_store(const tessel_checkpoint &c, const tessel_rows &x, void *stream)
{
    tessel_checkpoint cc = c;
    tessel_rows xx = x;
    void *args[] = {&cc, &xx};
#define KERNEL(T) ((const void *)store_kernel<T>)
    return launched(hipLaunchKernel(BY_TYPE(c.type, KERNEL), grid_of(c), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

int launch_restore(const tessel_checkpoint &c, const tessel_rows &x, void *stream)
{
    tessel_checkpoint cc = c;
    tessel_rows xx = x;
    void *args[] = {&cc, &xx};
#define KERNEL(T) ((const void *)restore_kernel<T>)
    return launched(hipLaunchKernel(BY_TYPE(c.type, KERNEL), grid_of(c), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

int launch_gated(int act, const tessel_rows &g, const tessel_rows &u, const tessel_rows &a, const tessel_checkpoint &kg,
                 const tessel_checkpoint &ku, void *stream)
{
    tessel_rows gg = g, uu = u, aa = a;
    tessel_checkpoint c = kg, d = ku;
    void *args[] = {&gg, &uu, &aa, &c, &d};
#define KERNEL(T) (act == TESSEL_SILU ? (const void *)gated_kernel<T, TESSEL_SILU> : (const void *)gated_kernel<T, TESSEL_GELU>)
    return launched(hipLaunchKernel(BY_TYPE(kg.type, KERNEL), grid_of(kg), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

int launch_gated_backward(int act, const tessel_rows &da, const tessel_checkpoint &kg, const tessel_checkpoint &ku, const tessel_rows &dg,
                          const tessel_rows &du, const tessel_rows &a, void *stream)
{
    tessel_rows dd = da, gg = dg, uu = du, aa = a;
    tessel_checkpoint c = kg, d = ku;
    void *args[] = {&dd, &c, &d, &gg, &uu, &aa};
#define KERNEL(T) (act == TESSEL_SILU ? (const void *)gated_backward_kernel<T, TESSEL_SILU> : (const void *)gated_backward_kernel<T, TESSEL_GELU>)
    return launched(hipLaunchKernel(BY_TYPE(kg.type, KERNEL), grid_of(kg), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

}  // namespace tessel
