// The norms of queries and keys for each head with the rotation by position, forward and backward (formulas: include/tessel_block_ops.h).
//
// A wave takes one head of a token, a lane up to two pairs of its channels; backward, waves go over many heads and add up the gradients of w.
#include "tessel_rows.h"

namespace tessel {

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct RotateLaunch {
    tessel_rotation a;
    float *parts;                // [parts][2][dim]: the gradients of wq and wk, by workgroup
    int    num_parts;
};

// the channels of pair p of a head; behind those that turn, channels are paired as they come
__device__ __forceinline__ void pair_at(const tessel_rotation &a, int p, int &lo, int &hi)
{
    const int half = a.turning / 2;
    if (p >= half) {
        lo = a.turning + p - half;
        hi = lo + a.dim / 2 - half;
    } else {
        lo = a.neighbours ? 2 * p : p;
        hi = a.neighbours ? 2 * p + 1 : p + half;
    }
}

__device__ __forceinline__ void turn_of(const tessel_rotation &a, int64_t token, int p, float &sine, float &cosine)
{
    sine = 0;
    cosine = 1;
    if (p >= a.turning / 2) return;
    const double position = a.index_type == TESSEL_I64 ? (double)((const int64_t *)a.position)[token] : (double)((const int32_t *)a.position)[token];
    const double turns = position * a.frequency[p] * 0.15915494309189535;        // angle / (2 pi)
    sincospif((float)(2.0 * (turns - rint(turns))), &sine, &cosine);
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateLaunch l)
{
    const tessel_rotation &a = l.a;
    const int all = a.heads + a.kv_heads, lane = threadIdx.x & 63, pairs = a.dim / 2;
    const int64_t n = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6), token = n / all;
    if (token >= a.tokens) return;
    const int head = (int)(n % all);
    const bool key = head >= a.heads;
    const tessel_heads &from = key ? a.k : a.q, &to = key ? a.k_out : a.q_out;
    const int h = key ? head - a.heads : head;
    const T *z = (const T *)from.data + token * from.token_stride + h * from.head_stride;
    T *o = (T *)to.data + token * to.token_stride + h * to.head_stride;
    const float *w = key ? a.wk : a.wq;
    float x[2] = {}, y[2] = {}, sum = 0;
    int lo[2], hi[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        pair_at(a, lane + 64 * i, lo[i], hi[i]);
        if (lane + 64 * i < pairs) {
            x[i] = (float)z[lo[i]];
            y[i] = (float)z[hi[i]];
        }
        sum += x[i] * x[i] + y[i] * y[i];
    }
    const float over = w ? 1.0f / sqrtf(wave_sum(sum) / a.dim + a.eps) : 1.0f;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        if (lane + 64 * i >= pairs) continue;
        float s, c;
        turn_of(a, token, lane + 64 * i, s, c);
        const float p = x[i] * over * (w ? w[lo[i]] : 1.0f), q = y[i] * over * (w ? w[hi[i]] : 1.0f);
        o[lo[i]] = (T)(p * c - q * s);
        o[hi[i]] = (T)(p * s + q * c);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void rotate_backward_kernel(RotateLaunch l)
{
    __shared__ float sums[kWaves][2][2][128];
    const tessel_rotation &a = l.a;
    const int all = a.heads + a.kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.dim / 2;
    float dw[2][2][2] = {};                                      // [q or k][pair][lo or hi]
    for (int64_t n = (int64_t)blockIdx.x * kWaves + wave; n < a.tokens * all; n += (int64_t)gridDim.x * kWaves) {
        const int64_t token = n / all;
        const int head = (int)(n % all);
        const bool key = head >= a.heads;
        const tessel_heads &from = key ? a.k : a.q, &grad = key ? a.dk_out : a.dq_out, &to = key ? a.dk : a.dq;
        const int h = key ? head - a.heads : head;
        const T *z = (const T *)from.data + token * from.token_stride + h * from.head_stride;
        const T *g = (const T *)grad.data + token * grad.token_stride + h * grad.head_stride;
        T *o = (T *)to.data + token * to.token_stride + h * to.head_stride;
        const float *w = key ? a.wk : a.wq;
        float x[2] = {}, y[2] = {}, dx[2] = {}, dy[2] = {}, sum = 0;
        int lo[2], hi[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            pair_at(a, lane + 64 * i, lo[i], hi[i]);
            if (lane + 64 * i < pairs) {
                x[i] = (float)z[lo[i]];
                y[i] = (float)z[hi[i]];
                const float p = (float)g[lo[i]], q = (float)g[hi[i]];
                float s, c;
                turn_of(a, token, lane + 64 * i, s, c);
                dx[i] = p * c + q * s;
                dy[i] = q * c - p * s;
            }
            sum += x[i] * x[i] + y[i] * y[i];
        }
        if (w) {
            const float over = 1.0f / sqrtf(wave_sum(sum) / a.dim + a.eps);
            sum = 0;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                if (lane + 64 * i >= pairs) continue;
                x[i] *= over;
                y[i] *= over;
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    dw[k][i][0] += key == (k == 1) ? dx[i] * x[i] : 0.0f;
                    dw[k][i][1] += key == (k == 1) ? dy[i] * y[i] : 0.0f;
                }
                dx[i] *= w[lo[i]];
                dy[i] *= w[hi[i]];
                sum += dx[i] * x[i] + dy[i] * y[i];
            }
            const float mean = wave_sum(sum) / a.dim;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                dx[i] = over * (dx[i] - x[i] * mean);
                dy[i] = over * (dy[i] - y[i] * mean);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
            if (lane + 64 * i < pairs) {
                o[lo[i]] = (T)dx[i];
                o[hi[i]] = (T)dy[i];
            }
    }
    if (!a.wq) return;
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < 2; j++) sums[wave][k][j][lane + 64 * i] = dw[k][i][j];
    __syncthreads();
    for (int n = threadIdx.x; n < 2 * a.dim; n += kThreads) {
        const int k = n / a.dim, j = n % a.dim / pairs, p = n % pairs;
        int lo, hi;
        pair_at(a, p, lo, hi);
        float sum = 0;
#pragma unroll
        for (int w = 0; w < kWaves; w++) sum += sums[w][k][j][p];
        l.parts[((int64_t)blockIdx.x * 2 + k) * a.dim + (j ? hi : lo)] = sum;
    }
}

// sums of the workgroups' parts: 64 channels a workgroup, sixteen waves over every sixteenth part each
__global__ __launch_bounds__(1024) void rotate_sum_kernel(RotateLaunch l)
{
    __shared__ float sums[16][64];
    const tessel_rotation &a = l.a;
    const int which = blockIdx.y, lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane, group = threadIdx.x >> 6;
    float sum = 0;
    if (col < a.dim)
#pragma unroll 8
        for (int p = group; p < l.num_parts; p += 16) sum += l.parts[((int64_t)p * 2 + which) * a.dim + col];
    sums[group][lane] = sum;
    __syncthreads();
    if (group != 0 || col >= a.dim) return;
    sum = 0;
#pragma unroll
    for (int g = 0; g < 16; g++) sum += sums[g][lane];
    float *out = (which == 0 ? a.dwq : a.dwk) + col;
    *out = a.accumulate ? *out + sum : sum;
}

int rotate_parts(const tessel_rotation &a)
{
    const int64_t all = a.tokens * (a.heads + a.kv_heads), groups = (all + kWaves - 1) / kWaves;
    return (int)(groups < 1024 ? groups : 1024);
}

int launch_rotate(const tessel_rotation &a, void *stream)
{
    RotateLaunch l = {a, nullptr, 0};
    void *args[] = {&l};
    const int64_t all = a.tokens * (a.heads + a.kv_heads), groups = (all + kWaves - 1) / kWaves;
#define KERNEL(T) ((const void *)rotate_kernel<T>)
    const void *kernel = a.type == TESSEL_BF16 ? KERNEL(bf16) : a.type == TESSEL_F16 ? KERNEL(f16) : KERNEL(float);
#undef KERNEL
    return launched(hipLaunchKernel(kernel, dim3((unsigned)groups), dim3(kThreads), args, 0, (hipStream_t)stream));
}

int launch_rotate_backward(const tessel_rotation &a, float *parts, void *stream)
{
    RotateLaunch l = {a, parts, rotate_parts(a)};
    void *args[] = {&l};
#define KERNEL(T) ((const void *)rotate_backward_kernel<T>)
    const void *kernel = a.type == TESSEL_BF16 ? KERNEL(bf16) : a.type == TESSEL_F16 ? KERNEL(f16) : KERNEL(float);
#undef KERNEL
    int e = 0;
    if (l.num_parts > 0) e = launched(hipLaunchKernel(kernel, dim3((unsigned)l.num_parts), dim3(kThreads), args, 0, (hipStream_t)stream));
    if (e == 0 && a.wq)
        e = launched(hipLaunchKernel((const void *)rotate_sum_kernel, dim3((unsigned)((a.dim + 63) / 64), 2), dim3(1024), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
