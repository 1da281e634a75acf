// The norms around a block with its gate and residual scale, forward and backward (formulas: include/tessel_block_ops.h).
//
// A row stays in the registers of its lanes from its one read to its one write: LANES lanes hold it, CHUNKS times eight channels each.
// Rows of up to 128 channels take 16 lanes, up to 512 a wave, longer ones up to 1024 lanes.  Workgroups go over many
// rows, so the parameters are read once a workgroup and their gradients are summed in registers, then over the rows a workgroup
// works on at once (LDS), then over the workgroups in the order of their numbers by a second kernel.
//
// Bound by memory: everything is read and written once.  8192 rows of 4096 bf16: forward 47 us (5.8 TB/s, part of it from the last cache),
// backward 86 us (4.7 TB/s, a large copy 4.8) and 6 us for the second kernel; 4 rows 4 us, a launch.  Rows of more than 8192 channels reach
// half of that (their registers do not last).
#include "tessel_rows.h"

namespace tessel {

struct NormLaunch {
    tessel_residual_norm a;
    float *parts;                // [parts][2][channels]: what the gradients of pre, and of post and the channels' gate, are made of, by workgroup
    int    num_parts;
};

// sum over a row's lanes; scratch: a word for each wave of the workgroup
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *scratch)
{
#pragma unroll
    for (int d = LANES < 64 ? LANES / 2 : 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        scratch += threadIdx.x / LANES * (LANES / 64);
        v = 0;
#pragma unroll
        for (int w = 0; w < LANES / 64; w++) v += scratch[w];
    }
    return v;
}

template <typename T>
__device__ __forceinline__ T *row_of(const tessel_rows &r, int64_t row) { return (T *)r.data + row * r.stride; }

template <int LANES> constexpr int threads_of() { return LANES > 256 ? LANES : 256; }

// The parameters of a lane's channels, ones for those that a call does not have (multiplying by them changes nothing, and one path through
// the kernels keeps their registers low).  They are kept in registers, in LDS (backward, two chunks: 48 registers less, of which there
// are then enough: 80 instead of 128 us for 8192 rows of 4096), or read again for each row (backward, more than 8192 channels, which LDS does not hold).
enum { kInRegisters, kInLds, kInMemory };
template <int LANES, int CHUNKS, int WHERE>
struct Parameters {
    static constexpr int kLds = WHERE == kInLds ? 3 * CHUNKS * 2 * LANES : 1;
    float kept[WHERE == kInRegisters ? 3 * CHUNKS : 1][8];
    const float *from[3];
    float4v *lds;
    __device__ __forceinline__ void read(float *v, int w, int k, int channels) const
    {
        if (from[w]) {
            load8<float>(v, from[w], 8 * ((int)threadIdx.x % LANES + k * LANES), channels);
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = 1.0f;
        }
    }
    __device__ __forceinline__ Parameters(const tessel_residual_norm &a, float4v *shared) : lds(shared + threadIdx.x % LANES)
    {
        from[0] = a.pre;
        from[1] = a.post;
        from[2] = a.gate_kind == TESSEL_GATE_CHANNEL ? (const float *)a.gate.data : nullptr;
        if constexpr (WHERE == kInRegisters) {
#pragma unroll
            for (int w = 0; w < 3; w++)
#pragma unroll
                for (int k = 0; k < CHUNKS; k++) read(kept[w * CHUNKS + k], w, k, a.channels);
        } else if constexpr (WHERE == kInLds) {
#pragma unroll
            for (int w = 0; w < 3; w++)
#pragma unroll
                for (int k = 0; k < CHUNKS; k++) {
                    float v[8];
                    read(v, w, k, a.channels);
                    lds[((w * CHUNKS + k) * 2) * LANES] = float4v{v[0], v[1], v[2], v[3]};
                    lds[((w * CHUNKS + k) * 2 + 1) * LANES] = float4v{v[4], v[5], v[6], v[7]};
                }
        }                                                        // (each lane reads back what it wrote itself)
    }
    __device__ __forceinline__ void get(float *v, int w, int k, int channels) const
    {
        if constexpr (WHERE == kInRegisters) {
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = kept[w * CHUNKS + k][j];
        } else if constexpr (WHERE == kInLds) {
            const float4v x = lds[((w * CHUNKS + k) * 2) * LANES], y = lds[((w * CHUNKS + k) * 2 + 1) * LANES];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                v[j] = x[j];
                v[4 + j] = y[j];
            }
        } else {
            read(v, w, k, channels);
        }
    }
};

// The rows of a workgroup: neighbours, so that a line of memory that two rows share is written through one cache (rows of 1000 channels,
// forward and backward: 163 us, with a workgroup's rows spread over the batch 180; rows of whole lines the same).
struct Range {
    int64_t begin, end;
    __device__ __forceinline__ Range(int64_t tokens, int rows)
    {
        const int64_t steps = (tokens + rows - 1) / rows, per = steps / gridDim.x, more = steps % gridDim.x, b = blockIdx.x;
        begin = (b * per + min(b, more)) * rows;
        end = min(begin + (per + (b < more ? 1 : 0)) * rows, tokens);
    }
};

// Eight values of a row, in their places behind settled().  Rows of up to 8192 channels are read without branches (32 Mi values of bf16, forward and
// backward: rows of 4095 157 us, in pieces behind a branch 192; of 1500 163 and 229; of 4096 138 both); longer ones have no registers
// left for it (10000 channels of 32 bits: 779 and 652).
template <typename T, int LANES>
__device__ __forceinline__ typename Eight<T>::type chunk8(const T *row, int col, int channels)
{
    if constexpr (LANES > 512) return raw8<T>(row, col, channels);
    else return take8<T, LANES == 16>(row, col, channels);
}
template <typename T, int LANES, bool TOKEN, typename... V>
__device__ __forceinline__ void settled(int col, int channels, typename Eight<T>::type &gate, V &...v)
{
    if constexpr (LANES > 512) return;
    else if constexpr (TOKEN) settle8<T, LANES == 16>(col, channels, v..., gate);
    else settle8<T, LANES == 16>(col, channels, v...);
}

// TOKEN: a gate for each token and channel
template <typename T, int LANES, int CHUNKS, bool TOKEN>
__global__ __launch_bounds__(threads_of<LANES>()) void norm_kernel(NormLaunch l)
{
    typedef Parameters<LANES, CHUNKS, kInRegisters> P;
    constexpr int kRows = threads_of<LANES>() / LANES;
    __shared__ float scratch[2][threads_of<LANES>() / 64];
    __shared__ float4v shared[P::kLds];
    const tessel_residual_norm &a = l.a;
    const int lane = threadIdx.x % LANES, C = a.channels;
    const P p(a, shared);
    const Range range(a.tokens, kRows);
    for (int64_t first = range.begin; first < range.end; first += kRows) {
        // (a workgroup's rows go through the barriers together; behind the last row, the last one once more without a write)
        const bool there = first + threadIdx.x / LANES < range.end;
        const int64_t row = there ? first + threadIdx.x / LANES : range.end - 1;
        const int begin = there ? 8 * lane : C;
        float x[CHUNKS][8], y[CHUNKS][8], sum = 0;
        typename Eight<T>::type rx[CHUNKS], ry[CHUNKS], rg[CHUNKS];
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = begin + 8 * k * LANES;
            rx[k] = chunk8<T, LANES>(row_of<T>(a.x, row), col, C);
            ry[k] = chunk8<T, LANES>(row_of<T>(a.y, row), col, C);
            if (TOKEN) rg[k] = chunk8<T, LANES>(row_of<T>(a.gate, row), col, C);
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = begin + 8 * k * LANES;
            settled<T, LANES, TOKEN>(col, C, rg[k], rx[k], ry[k]);
            widen8<T>(x[k], rx[k]);
            widen8<T>(y[k], ry[k]);
        }
        float over_y = 1.0f;
        if (a.post) {
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int j = 0; j < 8; j++) sum += y[k][j] * y[k][j];
            over_y = 1.0f / sqrtf(row_sum<LANES>(sum, scratch[0]) / a.channels + a.eps);
        }
        sum = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            float post[8], gate[8];
            p.get(post, 1, k, C);
            if (!TOKEN) p.get(gate, 2, k, C);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float u = y[k][j] * over_y * post[j];
                x[k][j] = a.scale * x[k][j] + (TOKEN ? (float)rg[k][j] : gate[j]) * u;
                sum += x[k][j] * x[k][j];
            }
            store8<T>(row_of<T>(a.r, row), x[k], begin + 8 * k * LANES, C);
        }
        const float over_r = 1.0f / sqrtf(row_sum<LANES>(sum, scratch[1]) / a.channels + a.eps);
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            float pre[8];
            p.get(pre, 0, k, C);
#pragma unroll
            for (int j = 0; j < 8; j++) x[k][j] *= over_r * pre[j];
            store8<T>(row_of<T>(a.h, row), x[k], begin + 8 * k * LANES, C);
        }
        if (lane == 0 && there) {
            a.stats[row] = over_y;
            a.stats[a.tokens + row] = over_r;
        }
        if constexpr (LANES > 64) __syncthreads();               // (scratch is free again)
    }
}

template <typename T, int LANES, int CHUNKS, bool TOKEN>
__global__ __launch_bounds__(threads_of<LANES>(), LANES > 512 || (LANES < 128 && sizeof(T) == 2) ? 4 : CHUNKS == 1 ? 3 : LANES > 256 || sizeof(T) == 4 ? 2 : 3) void norm_backward_kernel(NormLaunch l)
{
    typedef Parameters<LANES, CHUNKS, CHUNKS == 1 ? kInRegisters : LANES <= 512 ? kInLds : kInMemory> P;
    __shared__ float4v shared[P::kLds];
    constexpr int kRows = threads_of<LANES>() / LANES;
    __shared__ float scratch[2][threads_of<LANES>() / 64];
    const tessel_residual_norm &a = l.a;
    const int lane = threadIdx.x % LANES, C = a.channels;
    const P p(a, shared);
    // by: sum of r's gradient times y over its root mean square (of which the gradients of post and the channels' gate are multiples);
    // with TOKEN, times the gate, and so post's
    float dpre[CHUNKS][8] = {}, by[CHUNKS][8] = {};
    const Range range(a.tokens, kRows);
    for (int64_t first = range.begin; first < range.end; first += kRows) {
        const bool there = first + threadIdx.x / LANES < range.end;           // (as in norm_kernel)
        const int64_t row = there ? first + threadIdx.x / LANES : range.end - 1;
        const int begin = there ? 8 * lane : C;
        typename Eight<T>::type rx[CHUNKS], ry[CHUNKS], rr[CHUNKS], rh[CHUNKS], rg[CHUNKS];
        float x[CHUNKS][8], y[CHUNKS][8], dn[CHUNKS][8], sum = 0;
        const float over_y = a.stats[row], over_r = a.stats[a.tokens + row];
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = begin + 8 * k * LANES;
            rx[k] = chunk8<T, LANES>(row_of<T>(a.x, row), col, C);
            ry[k] = chunk8<T, LANES>(row_of<T>(a.y, row), col, C);
            rr[k] = chunk8<T, LANES>(row_of<T>(a.dr, row), col, C);
            rh[k] = chunk8<T, LANES>(row_of<T>(a.dh, row), col, C);
            if (TOKEN) rg[k] = chunk8<T, LANES>(row_of<T>(a.gate, row), col, C);
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = begin + 8 * k * LANES;
            settled<T, LANES, TOKEN>(col, C, rg[k], rx[k], ry[k], rr[k], rh[k]);
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            float pre[8], post[8], gate[8];
            p.get(pre, 0, k, C);
            p.get(post, 1, k, C);
            if (!TOKEN) p.get(gate, 2, k, C);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                y[k][j] = (float)ry[k][j] * over_y;
                const float u = y[k][j] * post[j];
                x[k][j] = (a.scale * (float)rx[k][j] + (TOKEN ? (float)rg[k][j] : gate[j]) * u) * over_r;      // r by its root mean square
                dn[k][j] = (float)rh[k][j];
                dpre[k][j] += dn[k][j] * x[k][j];
                dn[k][j] *= pre[j];
                sum += dn[k][j] * x[k][j];
            }
        }
        const float mean_r = row_sum<LANES>(sum, scratch[0]) / a.channels;
        sum = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int col = begin + 8 * k * LANES;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                dn[k][j] = (float)rr[k][j] + over_r * (dn[k][j] - x[k][j] * mean_r);      // the gradient of r
                v[j] = a.scale * dn[k][j];
            }
            store8<T>(row_of<T>(a.dx, row), v, col, C);
            float post[8], gate[8];
            p.get(post, 1, k, C);
            if (!TOKEN) p.get(gate, 2, k, C);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                if (TOKEN) {
                    v[j] = dn[k][j] * (y[k][j] * post[j]);
                    dn[k][j] *= (float)rg[k][j];
                }
                by[k][j] += dn[k][j] * y[k][j];
                dn[k][j] *= TOKEN ? post[j] : gate[j] * post[j];
                sum += dn[k][j] * y[k][j];
            }
            if (TOKEN) store8<T>(row_of<T>(a.dgate, row), v, col, C);
        }
        const float mean_y = a.post ? row_sum<LANES>(sum, scratch[1]) / a.channels : 0.0f;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++)
#pragma unroll
            for (int j = 0; j < 8; j++) dn[k][j] = over_y * (dn[k][j] - y[k][j] * mean_y);
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) store8<T>(row_of<T>(a.dy, row), dn[k], begin + 8 * k * LANES, C);
        if constexpr (LANES > 64) __syncthreads();
    }
    // the rows of a workgroup add up in order
    if constexpr (kRows > 1) {
        __shared__ float sums[(kRows - 1) * LANES * 8 * 2];
        static_assert(CHUNKS == 1, "one chunk a lane");
        const int group = threadIdx.x / LANES;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            float *at = sums + ((group - 1) * 16 + j) * LANES + lane;
            if (group > 0) {
                at[0] = dpre[0][j];
                at[8 * LANES] = by[0][j];
            }
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll 1
        for (int g = 0; g < kRows - 1; g++)
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float *at = sums + (g * 16 + j) * LANES + lane;
                dpre[0][j] += at[0];
                by[0][j] += at[8 * LANES];
            }
    }
    float *out = l.parts + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        const int col = 8 * (lane + k * LANES);
        store8<float>(out, dpre[k], col, C);
        store8<float>(out + C, by[k], col, C);
    }
}

// sums of the workgroups' parts: 64 columns a workgroup, sixteen waves over every sixteenth part each
__global__ __launch_bounds__(1024) void norm_sum_kernel(NormLaunch l)
{
    __shared__ float sums[16][64];
    const tessel_residual_norm &a = l.a;
    const int which = blockIdx.y, lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane, group = threadIdx.x >> 6;
    const bool gated = a.gate_kind == TESSEL_GATE_CHANNEL;
    if (which == 1 && !a.post && !gated) return;
    float sum = 0;
    if (col < a.channels)
#pragma unroll 8
        for (int p = group; p < l.num_parts; p += 16) sum += l.parts[((int64_t)p * 2 + which) * a.channels + col];
    sums[group][lane] = sum;
    __syncthreads();
    if (group != 0 || col >= a.channels) return;
    sum = 0;
#pragma unroll
    for (int g = 0; g < 16; g++) sum += sums[g][lane];
    const auto put = [&](float *out, float v) { out[col] = a.accumulate ? out[col] + v : v; };
    if (which == 0) {
        put(a.dpre, sum);
    } else {
        if (a.post) put(a.dpost, gated ? sum * ((const float *)a.gate.data)[col] : sum);
        if (gated) put(a.dgate_channel, a.post ? sum * a.post[col] : sum);
    }
}

struct NormShape {
    int lanes, chunks, threads, rows;
};
static NormShape shape_of(int channels)
{
    // (4096 channels: 256 lanes with two chunks; 512 with one meet at barriers of eight waves, 61 instead of 50 us forward for 8192 rows)
    const int lanes = channels <= 128 ? 16 : channels <= 512 ? 64 : channels <= 1024 ? 128 : channels <= 4096 ? 256 : channels <= 8192 ? 512 : 1024;
    const int threads = lanes > 256 ? lanes : 256;
    return {lanes, channels > lanes * 8 ? 2 : 1, threads, threads / lanes};
}

// workgroups: at most one for each row that they work on at once
static int64_t groups_of(const tessel_residual_norm &a, int64_t most)
{
    const NormShape s = shape_of(a.channels);
    const int64_t need = (a.tokens + s.rows - 1) / s.rows;
    return need < most ? need : most;
}

// backward: as many workgroups as are resident at once, each leaves a part.  More of them where reads of 16 bits are many small ones (rows of
// 4095 bf16: 193 instead of 216 us forward and backward, of 500: 238 instead of 264), fewer where a few waves keep memory busy (4096
// channels of bf16: 138 instead of 142).
int norm_parts(const tessel_residual_norm &a)
{
    const NormShape s = shape_of(a.channels);
    const bool half = a.type != TESSEL_F32;
    return (int)groups_of(a, s.threads > 256 ? 256 : s.chunks == 1 ? (half && s.lanes < 128 ? 1024 : 768) : half && a.channels % 8 ? 768 : 512);
}

template <typename T, bool TOKEN>
static const void *norm_of(const NormShape &s, bool back)
{
#define PICK(L, K) if (s.lanes == L && s.chunks == K) return back ? (const void *)norm_backward_kernel<T, L, K, TOKEN> : (const void *)norm_kernel<T, L, K, TOKEN>;
    PICK(16, 1)
    PICK(64, 1)
    PICK(128, 1)
    PICK(256, 1)
    PICK(256, 2)
    PICK(512, 2)
    PICK(1024, 2)
#undef PICK
    return nullptr;
}

template <bool TOKEN>
static const void *norm_of(const tessel_residual_norm &a, bool back)
{
    const NormShape s = shape_of(a.channels);
    return a.type == TESSEL_BF16 ? norm_of<bf16, TOKEN>(s, back) : a.type == TESSEL_F16 ? norm_of<f16, TOKEN>(s, back) : norm_of<float, TOKEN>(s, back);
}

static const void *norm_of(const tessel_residual_norm &a, bool back)
{
    return a.gate_kind == TESSEL_GATE_TOKEN ? norm_of<true>(a, back) : norm_of<false>(a, back);
}

int launch_norm(const tessel_residual_norm &a, void *stream)
{
    NormLaunch l = {a, nullptr, 0};
    void *args[] = {&l};
    const NormShape s = shape_of(a.channels);
    const int64_t groups = groups_of(a, s.threads > 256 ? 512 : 2048);
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
        e = launched(hipLaunchKernel(norm_of(a, true), dim3((unsigned)l.num_parts), dim3(s.threads), args, 0, (hipStream_t)stream));
    if (e == 0)
        e = launched(hipLaunchKernel((const void *)norm_sum_kernel, dim3((unsigned)((a.channels + 63) / 64), 2), dim3(1024), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
