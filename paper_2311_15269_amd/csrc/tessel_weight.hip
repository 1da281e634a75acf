// Gradient of a product's weights from an input kept in 8 bits: dw[n][c] = sum_t dy[t][n] x[t][c] (include/tessel_block_ops.h).
//
// A workgroup of four waves takes 128 x 128 of dw, 64 x 64 a wave, and goes over the tokens 64 at a time.  The summed index runs along
// the rows of both inputs, so both operands come out of LDS by transposing reads.  The checkpoint is turned into numbers
// of the matrix instruction's type on its way to LDS, which is exact.  Few tiles: the tokens are split over several workgroups,
// whose sums a second kernel adds in the order of their numbers.
#include "tessel_rows.h"

namespace tessel {

constexpr int kThreads = 256, kTile = 128, kSteps = 64;

struct WeightLaunch {
    tessel_weight_grad a;
    float  *parts;               // [splits][outputs][channels], or NULL: one split, straight to dw
    int     splits;
    int64_t per;                 // tokens a split, a multiple of kSteps
    int     tiles_c;
};

template <typename T>
struct DyStage {
    uint4v v[4];
    __device__ __forceinline__ void fetch(const tessel_weight_grad &a, int64_t t0, int64_t end, int n0)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = threadIdx.x + i * kThreads, col = n0 + 8 * (k % 16);
            const int64_t t = t0 + k / 16;
            typename Eight<T>::type w = {};
            if (t < end) {
                const T *row = (const T *)a.dy.data + t * a.dy.stride;
                if (col + 8 <= a.outputs) {
                    w = *(const typename Eight<T>::type *)(row + col);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; j++)
                        if (col + j < a.outputs) w[j] = row[col + j];
                }
            }
            v[i] = __builtin_bit_cast(uint4v, w);
        }
    }
    __device__ __forceinline__ void put(uint4v *tile) const
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = threadIdx.x + i * kThreads;
            tile[chunk_at<128>(k / 16, k % 16)] = v[i];
        }
    }
};

template <typename T>
struct HeldStage {
    uint2    v[4];
    uint32_t e[4];
    __device__ __forceinline__ void fetch(const tessel_weight_grad &a, int64_t t0, int64_t end, int c0)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = threadIdx.x + i * kThreads, col = c0 + 8 * (k % 16);
            const int64_t t = t0 + k / 16;
            v[i] = make_uint2(0, 0);
            e[i] = 1;
            if (t < end && col < a.x.channels) {
                v[i] = *(const uint2 *)(a.x.values + t * a.x.value_stride + col);
                e[i] = a.x.exponents[t * a.x.exponent_stride + col / kGroup];
            }
        }
    }
    __device__ __forceinline__ void put(uint4v *tile) const
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = threadIdx.x + i * kThreads;
            float f[8];
            held8(f, v[i], e[i]);
            uint4v w;
#pragma unroll
            for (int j = 0; j < 4; j++) w[j] = pack2<T>(f[2 * j], f[2 * j + 1]);
            tile[chunk_at<128>(k / 16, k % 16)] = w;
        }
    }
};

template <typename T>
__global__ __launch_bounds__(kThreads, 2) void weight_kernel(WeightLaunch l)
{
    __shared__ __attribute__((aligned(256))) uint4v rows[kSteps * kTile / 8], columns[kSteps * kTile / 8];
    const tessel_weight_grad &a = l.a;
    const int n0 = blockIdx.x / l.tiles_c * kTile, c0 = blockIdx.x % l.tiles_c * kTile;
    const int64_t begin = blockIdx.y * l.per, end = min(begin + l.per, a.x.tokens);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
    const int wn = wave >> 1, wc = wave & 1;
    const Reader<128> at;
    float16v acc[2][2] = {};
    DyStage<T> ds;
    HeldStage<T> hs;
    ds.fetch(a, begin, end, n0);
    hs.fetch(a, begin, end, c0);
    for (int64_t t = begin; t < end; t += kSteps) {
        __syncthreads();
        ds.put(rows);
        hs.put(columns);
        __syncthreads();
        ds.fetch(a, t + kSteps, end, n0);
        hs.fetch(a, t + kSteps, end, c0);
#pragma unroll
        for (int s = 0; s < kSteps / 16; s++) {
            uint4v x[2], y[2];
#pragma unroll
            for (int b = 0; b < 2; b++) {
                x[b] = at.columns((const lds_tile *)rows, 16 * s, 2 * wn + b);
                y[b] = at.columns((const lds_tile *)columns, 16 * s, 2 * wc + b);
            }
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int j = 0; j < 2; j++) acc[i][j] = mma<T>(x[i], y[j], acc[i][j]);
        }
    }
    float *out = l.parts ? l.parts + (int64_t)blockIdx.y * a.outputs * a.x.channels : a.dw;
    const int64_t stride = l.parts ? a.x.channels : a.dw_stride;
    const bool add = !l.parts && a.accumulate;
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const int c = c0 + 64 * wc + 32 * j + (lane & 31);
            if (c >= a.x.channels) continue;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const int n = n0 + 64 * wn + 32 * i + 8 * (r / 4) + 4 * half + r % 4;
                if (n >= a.outputs) continue;
                float *p = out + n * stride + c;
                *p = add ? *p + acc[i][j][r] : acc[i][j][r];
            }
        }
}

__global__ __launch_bounds__(kThreads) void weight_sum_kernel(WeightLaunch l)
{
    const tessel_weight_grad &a = l.a;
    const int64_t size = (int64_t)a.outputs * a.x.channels;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < size; i += (int64_t)gridDim.x * kThreads) {
        float *p = a.dw + i / a.x.channels * a.dw_stride + i % a.x.channels;
        float sum = a.accumulate ? *p : 0.0f;
        for (int s = 0; s < l.splits; s++) sum += l.parts[s * size + i];
        *p = sum;
    }
}

static int64_t tiles_of(const tessel_weight_grad &a)
{
    return (int64_t)((a.outputs + kTile - 1) / kTile) * ((a.x.channels + kTile - 1) / kTile);
}

// splits of the tokens: until 512 workgroups are there (two a compute unit), none shorter than 256 tokens
int weight_parts(const tessel_weight_grad &a)
{
    const int64_t tiles = tiles_of(a), most = (a.x.tokens + 255) / 256, want = tiles > 0 ? 512 / tiles : 1;
    const int64_t s = want < most ? want : most;
    return s < 1 ? 1 : (int)s;
}

int launch_weight_gradient(const tessel_weight_grad &a, float *parts, void *stream)
{
    WeightLaunch l = {a, nullptr, weight_parts(a), 0, (a.x.channels + kTile - 1) / kTile};
    l.per = ((a.x.tokens + l.splits - 1) / l.splits + kSteps - 1) / kSteps * kSteps;
    if (l.splits > 1) l.parts = parts;
    void *args[] = {&l};
    const void *kernel = a.x.type == TESSEL_BF16 ? (const void *)weight_kernel<bf16> : (const void *)weight_kernel<f16>;
    int e = launched(hipLaunchKernel(kernel, dim3((unsigned)tiles_of(a), (unsigned)l.splits), dim3(kThreads), args, 0, (hipStream_t)stream));
    if (e == 0 && l.parts)
        e = launched(hipLaunchKernel((const void *)weight_sum_kernel, dim3(1024), dim3(kThreads), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
