// The norms around a block with its gate and residual scale, forward and backward (formulas: include/tessel_block_ops.h).
//
// A row stays in the registers of its lanes from its one read to its one write: LANES lanes hold it, CHUNKS chunks of eight channels each.
// Rows of up to 1024 channels take a wave (four rows a workgroup and no barrier), longer ones a workgroup.  Workgroups go over many
// rows, so the parameters are read once a workgroup and their gradients are summed in registers, then over the workgroups
// in the order of their numbers by a second kernel.
#include "tessel_rows.h"

namespace tessel {

struct NormLaunch {
    tessel_residual_norm a;
    float *parts;                // [parts][3][channels]: gradients of pre, post and the channels' gate, by workgroup
    int    num_parts;
};

template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *scratch)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < LANES / 64; w++) v += scratch[w];
    }
    return v;
}

template <typename T>
__device__ __forceinline__ T *row_of(const tessel_rows &r, int64_t row) { return (T *)r.data + row * r.stride; }

template <int LANES> constexpr int threads_of() { return LANES > 64 ? LANES : 256; }

template <typename T, int LANES, int CHUNKS>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_kernel(NormLaunch l)
{
    constexpr int kRows = threads_of<LANES>() / LANES;
    __shared__ float scratch[2][LANES > 64 ? LANES / 64 : 1];
    const tessel_residual_norm &a = l.a;
    const int lane = threadIdx.x % LANES, C = a.channels;
    float pre[CHUNKS][8], post[CHUNKS][8], gate[CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        const int col = 8 * (lane + k * LANES);
        load8<float>(pre[k], a.pre, col, C);
        if (a.post) load8<float>(post[k], a.post, col, C);
        if (a.gate_kind == TESSEL_GATE_CHANNEL) load8<float>(gate[k], (const float *)a.gate.data, col, C);
    }
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.tokens; row += (int64_t)gridDim.x * kRows) {
        float x[CHUNKS][8], y[CHUNKS][8], sum = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = 8 * (lane + k * LANES);
            load8<T>(x[k], row_of<T>(a.x, row), col, C);
            load8<T>(y[k], row_of<T>(a.y, row), col, C);
            if (a.gate_kind == TESSEL_GATE_TOKEN) load8<T>(gate[k], row_of<T>(a.gate, row), col, C);
        }
        float over_y = 1.0f;
        if (a.post) {
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int j = 0; j < 8; j++) sum += y[k][j] * y[k][j];
            over_y = 1.0f / sqrtf(row_sum<LANES>(sum, scratch[0]) / C + a.eps);
        }
        sum = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                float u = y[k][j];
                if (a.post) u = u * over_y * post[k][j];
                if (a.gate_kind != TESSEL_GATE_NONE) u *= gate[k][j];
                x[k][j] = a.scale * x[k][j] + u;
                sum += x[k][j] * x[k][j];
            }
            store8<T>(row_of<T>(a.r, row), x[k], 8 * (lane + k * LANES), C);
        }
        const float over_r = 1.0f / sqrtf(row_sum<LANES>(sum, scratch[1]) / C + a.eps);
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
#pragma unroll
            for (int j = 0; j < 8; j++) x[k][j] *= over_r * pre[k][j];
            store8<T>(row_of<T>(a.h, row), x[k], 8 * (lane + k * LANES), C);
        }
        if (lane == 0) {
            a.stats[row] = over_y;
            a.stats[a.tokens + row] = over_r;
        }
        if constexpr (LANES > 64) __syncthreads();               // (scratch is free again)
    }
}

template <typename T, int LANES, int CHUNKS>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_backward_kernel(NormLaunch l)
{
    constexpr int kRows = threads_of<LANES>() / LANES;
    __shared__ float scratch[2][LANES > 64 ? LANES / 64 : 1];
    const tessel_residual_norm &a = l.a;
    const int lane = threadIdx.x % LANES, C = a.channels;
    float pre[CHUNKS][8], post[CHUNKS][8], gate[CHUNKS][8], dpre[CHUNKS][8] = {}, dpost[CHUNKS][8] = {}, dgate[CHUNKS][8] = {};
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        const int col = 8 * (lane + k * LANES);
        load8<float>(pre[k], a.pre, col, C);
        if (a.post) load8<float>(post[k], a.post, col, C);
        if (a.gate_kind == TESSEL_GATE_CHANNEL) load8<float>(gate[k], (const float *)a.gate.data, col, C);
    }
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.tokens; row += (int64_t)gridDim.x * kRows) {
        float x[CHUNKS][8], y[CHUNKS][8], dr[CHUNKS][8], dh[CHUNKS][8], sum = 0;
        const float over_y = a.stats[row], over_r = a.stats[a.tokens + row];
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = 8 * (lane + k * LANES);
            load8<T>(x[k], row_of<T>(a.x, row), col, C);
            load8<T>(y[k], row_of<T>(a.y, row), col, C);
            load8<T>(dr[k], row_of<T>(a.dr, row), col, C);
            load8<T>(dh[k], row_of<T>(a.dh, row), col, C);
            if (a.gate_kind == TESSEL_GATE_TOKEN) load8<T>(gate[k], row_of<T>(a.gate, row), col, C);
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++)
#pragma unroll
            for (int j = 0; j < 8; j++) {
                if (a.post) y[k][j] *= over_y;
                float u = a.post ? y[k][j] * post[k][j] : y[k][j];
                if (a.gate_kind != TESSEL_GATE_NONE) u *= gate[k][j];
                x[k][j] = (a.scale * x[k][j] + u) * over_r;      // r by its root mean square
                dpre[k][j] += dh[k][j] * x[k][j];
                dh[k][j] *= pre[k][j];
                sum += dh[k][j] * x[k][j];
            }
        const float mean_r = row_sum<LANES>(sum, scratch[0]) / C;
        sum = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = 8 * (lane + k * LANES);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                dr[k][j] += over_r * (dh[k][j] - x[k][j] * mean_r);
                x[k][j] = a.scale * dr[k][j];
            }
            store8<T>(row_of<T>(a.dx, row), x[k], col, C);
            if (a.gate_kind != TESSEL_GATE_NONE) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float u = a.post ? y[k][j] * post[k][j] : y[k][j];
                    x[k][j] = dr[k][j] * u;
                    dgate[k][j] += x[k][j];
                    dr[k][j] *= gate[k][j];
                }
                if (a.gate_kind == TESSEL_GATE_TOKEN) store8<T>(row_of<T>(a.dgate, row), x[k], col, C);
            }
            if (a.post) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    dpost[k][j] += dr[k][j] * y[k][j];
                    dr[k][j] *= post[k][j];
                    sum += dr[k][j] * y[k][j];
                }
            }
        }
        if (a.post) {
            const float mean_y = row_sum<LANES>(sum, scratch[1]) / C;
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int j = 0; j < 8; j++) dr[k][j] = over_y * (dr[k][j] - y[k][j] * mean_y);
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) store8<T>(row_of<T>(a.dy, row), dr[k], 8 * (lane + k * LANES), C);
        if constexpr (LANES > 64) __syncthreads();
    }
    float *out = l.parts + (int64_t)(blockIdx.x * kRows + threadIdx.x / LANES) * 3 * C;
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        const int col = 8 * (lane + k * LANES);
        store8<float>(out, dpre[k], col, C);
        if (a.post) store8<float>(out + C, dpost[k], col, C);
        if (a.gate_kind == TESSEL_GATE_CHANNEL) store8<float>(out + 2 * C, dgate[k], col, C);
    }
}

// sums of the workgroups' parts: 32 columns a workgroup, eight lanes a column over every eighth part
__global__ __launch_bounds__(256) void norm_sum_kernel(NormLaunch l)
{
    __shared__ float sums[8][32];
    const tessel_residual_norm &a = l.a;
    const int which = blockIdx.y, col = blockIdx.x * 32 + (threadIdx.x & 31), group = threadIdx.x >> 5;
    float *out = which == 0 ? a.dpre : which == 1 ? a.dpost : a.dgate_channel;
    if (which == 1 && !a.post) return;
    if (which == 2 && a.gate_kind != TESSEL_GATE_CHANNEL) return;
    float sum = 0;
    if (col < a.channels)
        for (int p = group; p < l.num_parts; p += 8) sum += l.parts[((int64_t)p * 3 + which) * a.channels + col];
    sums[group][threadIdx.x & 31] = sum;
    __syncthreads();
    if (group == 0 && col < a.channels) {
        sum = a.accumulate ? out[col] : 0.0f;
#pragma unroll
        for (int g = 0; g < 8; g++) sum += sums[g][threadIdx.x];
        out[col] = sum;
    }
}

struct NormShape {
    int lanes, chunks, threads, rows;
};
static NormShape shape_of(int channels)
{
    const int lanes = channels <= 1024 ? 64 : channels <= 4096 ? 256 : 1024;
    const int chunks = channels <= lanes * 8 ? 1 : 2;
    const int threads = lanes > 64 ? lanes : 256;
    return {lanes, chunks, threads, threads / lanes};
}

// workgroups: as many as are resident at once, at most one for each row (or four)
static int64_t groups_of(const tessel_residual_norm &a, int64_t most)
{
    const NormShape s = shape_of(a.channels);
    const int64_t need = (a.tokens + s.rows - 1) / s.rows;
    return need < most ? need : most;
}

int norm_parts(const tessel_residual_norm &a)
{
    const NormShape s = shape_of(a.channels);
    return (int)(groups_of(a, s.threads == 1024 ? 256 : 512) * s.rows);
}

template <typename T>
static const void *norm_of(const NormShape &s, bool back)
{
#define PICK(L, K) if (s.lanes == L && s.chunks == K) return back ? (const void *)norm_backward_kernel<T, L, K> : (const void *)norm_kernel<T, L, K>;
    PICK(64, 1)
    PICK(64, 2)
    PICK(256, 1)
    PICK(256, 2)
    PICK(1024, 1)
    PICK(1024, 2)
#undef PICK
    return nullptr;
}

static const void *norm_of(const tessel_residual_norm &a, bool back)
{
    const NormShape s = shape_of(a.channels);
    return a.type == TESSEL_BF16 ? norm_of<bf16>(s, back) : a.type == TESSEL_F16 ? norm_of<f16>(s, back) : norm_of<float>(s, back);
}

int launch_norm(const tessel_residual_norm &a, void *stream)
{
    NormLaunch l = {a, nullptr, 0};
    void *args[] = {&l};
    const NormShape s = shape_of(a.channels);
    const int64_t groups = groups_of(a, s.threads == 1024 ? 512 : 2048);
    if (groups == 0) return 0;
    return launched(hipLaunchKernel(norm_of(a, false), dim3((unsigned)groups), dim3(s.threads), args, 0, (hipStream_t)stream));
}

int launch_norm_backward(const tessel_residual_norm &a, float *parts, void *stream)
{
    NormLaunch l = {a, parts, norm_parts(a)};
    void *args[] = {&l};
    const NormShape s = shape_of(a.channels);
    int e = 0;
    if (l.num_parts > 0)
        e = launched(hipLaunchKernel(norm_of(a, true), dim3((unsigned)(l.num_parts / s.rows)), dim3(s.threads), args, 0, (hipStream_t)stream));
    if (e == 0)
        e = launched(hipLaunchKernel((const void *)norm_sum_kernel, dim3((unsigned)((a.channels + 31) / 32), 3), dim3(256), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
