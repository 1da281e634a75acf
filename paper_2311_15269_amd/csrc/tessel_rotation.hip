// The norms of queries and keys for each head with the rotation by position, forward and backward (formulas: include/tessel_block_ops.h).
//
// A head's pairs of channels lie in the registers of a group of lanes, VALUES pairs a lane, from its one read to its one write; a wave takes as many heads of a
// token as it has groups, several tokens where these have few heads, and goes on to the next heads.  The sines and cosines of its tokens
// it works out first, one a lane, and passes them around through LDS: all heads of a token share them.  Backward, a lane adds up the
// gradients of w for its channels over all that its wave goes over; then groups, waves and, by a second kernel, workgroups, in order.
#include <algorithm>

#include "tessel_rows.h"

namespace tessel {

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct RotateLaunch {
    tessel_rotation a;
    float   *parts;              // [parts][2][dim]: the gradients of wq and wk, by workgroup
    int32_t  num_parts;
    int32_t  group;              // lanes of a head: 2^group
    int32_t  heads;              // of a token that a wave takes at once: 2^heads
    int32_t  steps_q, steps;     // of those, for the queries, and for all heads of a token
    int32_t  splits;             // waves that share a token's steps
    int64_t  units;              // waves' turns in all
};

template <typename T, int V> struct Some {
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <typename T> struct Some<T, 1> {
    typedef T type;
};

// sum over the group of lanes; all of them get the same bits
template <int CTRL>
__device__ __forceinline__ float plus_lane(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 15, 15, true));
}
__device__ __forceinline__ float group_sum(float v, int group)
{
    if (group > 0) v = plus_lane<0xB1>(v);                       // neighbours
    if (group > 1) v = plus_lane<0x4E>(v);                       // pairs of a quad
    if (group > 2) v = plus_lane<0x141>(v);                      // quads of eight lanes, mirrored
    if (group > 3) v = plus_lane<0x140>(v);                      // halves of sixteen
    if (group > 4) v += __shfl_xor(v, 16);
    if (group > 5) v += __shfl_xor(v, 32);
    return v;
}

// sines and cosines of a wave's tokens, for all pairs of a head (those that do not turn: by no angle)
__device__ __forceinline__ void angles(const tessel_rotation &a, int64_t token, int tokens, float *cosine, float *sine)
{
    const int pairs = a.dim / 2, half = a.turning / 2;
    for (int i = threadIdx.x & 63; i < tokens * pairs; i += 64) {
        const int t = i / pairs, p = i - t * pairs;
        float s = 0.0f, c = 1.0f;
        if (p < half) {
            const int64_t n = min(token + t, a.tokens - 1);
            const double position = a.index_type == TESSEL_I64 ? (double)((const int64_t *)a.position)[n] : (double)((const int32_t *)a.position)[n];
            const double turns = position * a.frequency[p] * 0.15915494309189535;        // angle / (2 pi)
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        }
        cosine[i] = c;
        sine[i] = s;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // (the wave's own LDS: no barrier)
}

// What a lane has of a head: channels first[k] .. + V - 1 and second[k] .. + V - 1 of chunk k.  Pairs are the j-th of both; with `neighbours`, of which a chunk's
// channels are 2 V in a row, two in a row.
template <int V, int CHUNKS>
struct Mine {
    int  first[CHUNKS], second[CHUNKS], pair[CHUNKS];
    bool on[CHUNKS];
    __device__ __forceinline__ Mine(const tessel_rotation &a, int lane, int lanes)
    {
        const int chunks = a.dim / (2 * V), half = a.turning / 2;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int c = lane + k * lanes;
            on[k] = c < chunks;
            pair[k] = V * min(c, chunks - 1);
            const bool apart = pair[k] < half && !a.neighbours;
            first[k] = apart ? pair[k] : 2 * pair[k];
            second[k] = apart ? pair[k] + half : 2 * pair[k] + V;
        }
    }
};
template <typename T, int V>
__device__ __forceinline__ void spread(float *v, const typename Some<T, V>::type &x)
{
    if constexpr (V == 1) v[0] = (float)x;
    else
#pragma unroll
        for (int j = 0; j < V; j++) v[j] = (float)x[j];
}
template <typename T, int V>
__device__ __forceinline__ void put(T *to, const float *v)
{
    typename Some<T, V>::type x;
    if constexpr (V == 1) x = (T)v[0];
    else
#pragma unroll
        for (int j = 0; j < V; j++) x[j] = (T)v[j];
    *(typename Some<T, V>::type *)to = x;
}
template <int V>
__device__ __forceinline__ void get(float *v, const float *from)
{
#pragma unroll
    for (int j = 0; j < V; j++) v[j] = from[j];
}

// x and y turned by the angles, or with SIGN -1 back
template <int V, int SIGN>
__device__ __forceinline__ void turn(float *x, float *y, const float *c, const float *s, bool neighbours)
{
    const auto pair = [](float &a, float &b, float c, float s) {
        const float p = a, q = b;
        a = SIGN > 0 ? p * c - q * s : p * c + q * s;
        b = SIGN > 0 ? p * s + q * c : q * c - p * s;
    };
    if (V > 1 && neighbours) {
#pragma unroll
        for (int j = 0; j < V; j++) {
            float *z = j < V / 2 ? x + 2 * j : y + 2 * j - V;
            pair(z[0], z[1], c[j], s[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; j++) pair(x[j], y[j], c[j], s[j]);
    }
}

// A wave's turn: tokens, and steps over their heads
struct Turn {
    int64_t token;
    int     begin, end;
    __device__ __forceinline__ Turn(const RotateLaunch &l, int64_t unit, int tokens)
    {
        const int64_t group = unit / l.splits;
        const int part = (int)(unit - group * l.splits), per = (l.steps + l.splits - 1) / l.splits;
        token = group * tokens;
        begin = part * per;
        end = min(begin + per, l.steps);
    }
};

// the pointer to a head of a token, and its stride, by element
template <typename T>
__device__ __forceinline__ T *head_at(const tessel_heads &h, int64_t token, int head) { return (T *)h.data + token * h.token_stride + head * h.head_stride; }

template <typename T, int V, int CHUNKS>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateLaunch l)
{
    __shared__ __attribute__((aligned(16))) float table[kWaves][2][64 * V * CHUNKS];
    const tessel_rotation &a = l.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tokens = 64 >> l.group >> l.heads;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave;
    if (unit >= l.units) return;
    const Turn at(l, unit, tokens);
    const Mine<V, CHUNKS> mine(a, lane & ((1 << l.group) - 1), 1 << l.group);
    const int slot = lane >> l.group, head = slot & ((1 << l.heads) - 1), which = slot >> l.heads;
    const bool there = at.token + which < a.tokens;
    const int64_t token = min(at.token + which, a.tokens - 1);
    angles(a, at.token, tokens, table[wave][0], table[wave][1]);
    float c[CHUNKS][V], s[CHUNKS][V], w[CHUNKS][2][V];
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        get<V>(c[k], table[wave][0] + which * (a.dim / 2) + mine.pair[k]);
        get<V>(s[k], table[wave][1] + which * (a.dim / 2) + mine.pair[k]);
    }
    for (int step = at.begin; step < at.end; step++) {
        const bool key = step >= l.steps_q;
        const int n = ((key ? step - l.steps_q : step) << l.heads) + head, all = key ? a.kv_heads : a.heads;
        const T *z = head_at<const T>(key ? a.k : a.q, token, min(n, all - 1));
        float x[CHUNKS][V], y[CHUNKS][V], sum = 0;
        typename Some<T, V>::type rx[CHUNKS], ry[CHUNKS];
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            rx[k] = *(const typename Some<T, V>::type *)(z + mine.first[k]);
            ry[k] = *(const typename Some<T, V>::type *)(z + mine.second[k]);
        }
        if (a.wq && (step == at.begin || step == l.steps_q)) {
            const float *from = key ? a.wk : a.wq;
#pragma unroll
            for (int k = 0; k < CHUNKS; k++) {
                get<V>(w[k][0], from + mine.first[k]);
                get<V>(w[k][1], from + mine.second[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            spread<T, V>(x[k], rx[k]);
            spread<T, V>(y[k], ry[k]);
        }
        if (a.wq) {
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int j = 0; j < V; j++) sum += mine.on[k] ? x[k][j] * x[k][j] + y[k][j] * y[k][j] : 0.0f;
            const float over = 1.0f / sqrtf(group_sum(sum, l.group) / a.dim + a.eps);
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int j = 0; j < V; j++) {
                    x[k][j] *= over * w[k][0][j];
                    y[k][j] *= over * w[k][1][j];
                }
        }
        T *o = head_at<T>(key ? a.k_out : a.q_out, token, min(n, all - 1));
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            turn<V, 1>(x[k], y[k], c[k], s[k], a.neighbours && mine.pair[k] < a.turning / 2);
            if (there && n < all && mine.on[k]) {
                put<T, V>(o + mine.first[k], x[k]);
                put<T, V>(o + mine.second[k], y[k]);
            }
        }
    }
}

template <typename T, int V, int CHUNKS>
__global__ __launch_bounds__(kThreads) void rotate_backward_kernel(RotateLaunch l)
{
    __shared__ __attribute__((aligned(16))) float table[kWaves][2][64 * V * CHUNKS];
    __shared__ float sums[kWaves][2][256];
    const tessel_rotation &a = l.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tokens = 64 >> l.group >> l.heads;
    const Mine<V, CHUNKS> mine(a, lane & ((1 << l.group) - 1), 1 << l.group);
    const int slot = lane >> l.group, head = slot & ((1 << l.heads) - 1), which = slot >> l.heads;
    float dw[2][CHUNKS][2][V] = {}, w[CHUNKS][2][V];
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < l.units; unit += (int64_t)gridDim.x * kWaves) {
        const Turn at(l, unit, tokens);
        const bool there = at.token + which < a.tokens;
        const int64_t token = min(at.token + which, a.tokens - 1);
        angles(a, at.token, tokens, table[wave][0], table[wave][1]);
        float c[CHUNKS][V], s[CHUNKS][V];
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            get<V>(c[k], table[wave][0] + which * (a.dim / 2) + mine.pair[k]);
            get<V>(s[k], table[wave][1] + which * (a.dim / 2) + mine.pair[k]);
        }
        for (int step = at.begin; step < at.end; step++) {
            const bool key = step >= l.steps_q;
            const int n = ((key ? step - l.steps_q : step) << l.heads) + head, all = key ? a.kv_heads : a.heads;
            const bool mine_too = there && n < all;
            const T *z = head_at<const T>(key ? a.k : a.q, token, min(n, all - 1)), *g = head_at<const T>(key ? a.dk_out : a.dq_out, token, min(n, all - 1));
            float x[CHUNKS][V], y[CHUNKS][V], dx[CHUNKS][V], dy[CHUNKS][V], sum = 0;
            typename Some<T, V>::type rx[CHUNKS], ry[CHUNKS], gx[CHUNKS], gy[CHUNKS];
#pragma unroll
            for (int k = 0; k < CHUNKS; k++) {
                rx[k] = *(const typename Some<T, V>::type *)(z + mine.first[k]);
                ry[k] = *(const typename Some<T, V>::type *)(z + mine.second[k]);
                gx[k] = *(const typename Some<T, V>::type *)(g + mine.first[k]);
                gy[k] = *(const typename Some<T, V>::type *)(g + mine.second[k]);
            }
            if (a.wq && (step == at.begin || step == l.steps_q)) {
                const float *from = key ? a.wk : a.wq;
#pragma unroll
                for (int k = 0; k < CHUNKS; k++) {
                    get<V>(w[k][0], from + mine.first[k]);
                    get<V>(w[k][1], from + mine.second[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < CHUNKS; k++) {
                spread<T, V>(x[k], rx[k]);
                spread<T, V>(y[k], ry[k]);
                spread<T, V>(dx[k], gx[k]);
                spread<T, V>(dy[k], gy[k]);
                turn<V, -1>(dx[k], dy[k], c[k], s[k], a.neighbours && mine.pair[k] < a.turning / 2);
            }
            if (a.wq) {
#pragma unroll
                for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                    for (int j = 0; j < V; j++) sum += mine.on[k] ? x[k][j] * x[k][j] + y[k][j] * y[k][j] : 0.0f;
                const float over = 1.0f / sqrtf(group_sum(sum, l.group) / a.dim + a.eps);
                sum = 0;
                // (heads and channels that are not there count nothing)
                const auto add = [&](float (&to)[CHUNKS][2][V]) {
#pragma unroll
                    for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                        for (int j = 0; j < V; j++) {
                            x[k][j] *= over;
                            y[k][j] *= over;
                            to[k][0][j] += mine_too ? dx[k][j] * x[k][j] : 0.0f;
                            to[k][1][j] += mine_too ? dy[k][j] * y[k][j] : 0.0f;
                            dx[k][j] *= w[k][0][j];
                            dy[k][j] *= w[k][1][j];
                            sum += mine.on[k] ? dx[k][j] * x[k][j] + dy[k][j] * y[k][j] : 0.0f;
                        }
                };
                if (key) add(dw[1]);
                else add(dw[0]);
                const float mean = group_sum(sum, l.group) / a.dim;
#pragma unroll
                for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        dx[k][j] = over * (dx[k][j] - x[k][j] * mean);
                        dy[k][j] = over * (dy[k][j] - y[k][j] * mean);
                    }
            }
            T *o = head_at<T>(key ? a.dk : a.dq, token, min(n, all - 1));
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
                if (mine_too && mine.on[k]) {
                    put<T, V>(o + mine.first[k], dx[k]);
                    put<T, V>(o + mine.second[k], dy[k]);
                }
        }
    }
    if (!a.wq) return;
    // groups of a wave, waves of the workgroup
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int k = 0; k < CHUNKS; k++)
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int j = 0; j < V; j++) {
                    float v = dw[i][k][h][j];
                    for (int d = 1 << l.group; d < 64; d <<= 1) v += __shfl_xor(v, d);
                    if (slot == 0 && mine.on[k]) sums[wave][i][(h ? mine.second[k] : mine.first[k]) + j] = v;
                }
    __syncthreads();
    for (int n = threadIdx.x; n < 2 * a.dim; n += kThreads) {
        const int i = n >= a.dim, ch = n - i * a.dim;
        float sum = 0;
#pragma unroll
        for (int v = 0; v < kWaves; v++) sum += sums[v][i][ch];
        l.parts[(int64_t)blockIdx.x * 2 * a.dim + n] = sum;
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

// pairs a lane: eight or four where no chunk of them lies across the end of those that turn, else one
static int values_of(const tessel_rotation &a)
{
    const int turns = a.turning / 2, stays = (a.dim - a.turning) / 2;
    return turns % 8 == 0 && stays % 8 == 0 ? 8 : turns % 4 == 0 && stays % 4 == 0 ? 4 : 1;
}

static RotateLaunch rotate_launch(const tessel_rotation &a)
{
    RotateLaunch l = {};
    l.a = a;
    const int chunks = a.dim / (2 * values_of(a));
    while (l.group < 6 && 1 << l.group < chunks) l.group++;
    while (l.heads < 6 - l.group && 1 << l.heads < a.heads) l.heads++;
    const int each = 1 << l.heads, tokens = 64 >> l.group >> l.heads;
    l.steps_q = (a.heads + each - 1) / each;
    l.steps = l.steps_q + (a.kv_heads + each - 1) / each;
    // a wave for all heads of its tokens, or where that leaves the GPU idle, for fewer
    const int64_t groups = (a.tokens + tokens - 1) / tokens;
    l.splits = (int)std::min<int64_t>(l.steps, std::max<int64_t>(1, 4096 / std::max<int64_t>(1, groups)));
    l.splits = (l.steps + (l.steps + l.splits - 1) / l.splits - 1) / ((l.steps + l.splits - 1) / l.splits);       // (none without a step)
    l.units = groups * l.splits;
    return l;
}

int rotate_parts(const tessel_rotation &a) { return (int)std::min<int64_t>((rotate_launch(a).units + kWaves - 1) / kWaves, 1024); }

template <typename T>
static const void *rotate_of(const tessel_rotation &a, bool back)
{
#define PICK(V, K) (back ? (const void *)rotate_backward_kernel<T, V, K> : (const void *)rotate_kernel<T, V, K>)
    const int v = values_of(a);
    return v == 8 ? PICK(8, 1) : v == 4 ? PICK(4, 1) : a.dim > 128 ? PICK(1, 2) : PICK(1, 1);
#undef PICK
}
static const void *rotate_of(const tessel_rotation &a, bool back)
{
    return a.type == TESSEL_BF16 ? rotate_of<bf16>(a, back) : a.type == TESSEL_F16 ? rotate_of<f16>(a, back) : rotate_of<float>(a, back);
}

int launch_rotate(const tessel_rotation &a, void *stream)
{
    RotateLaunch l = rotate_launch(a);
    void *args[] = {&l};
    return launched(hipLaunchKernel(rotate_of(a, false), dim3((unsigned)((l.units + kWaves - 1) / kWaves)), dim3(kThreads), args, 0, (hipStream_t)stream));
}

int launch_rotate_backward(const tessel_rotation &a, float *parts, void *stream)
{
    RotateLaunch l = rotate_launch(a);
    l.parts = parts;
    l.num_parts = rotate_parts(a);
    void *args[] = {&l};
    int e = 0;
    if (l.num_parts > 0) e = launched(hipLaunchKernel(rotate_of(a, true), dim3((unsigned)l.num_parts), dim3(kThreads), args, 0, (hipStream_t)stream));
    if (e == 0 && a.wq)
        e = launched(hipLaunchKernel((const void *)rotate_sum_kernel, dim3((unsigned)((a.dim + 63) / 64), 2), dim3(1024), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
