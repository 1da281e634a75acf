// Causal attention over packed sequences with grouped heads, forward and backward (formulas: include/tessel_block_ops.h).
//
// A workgroup of four waves takes 128 queries of one head (or, for the gradients of k and v, 128 keys of a key-value head), 32 a wave.  All
// products are 32 x 32 x 16 matrix instructions, arranged so that a lane of the score tile holds ONE query (key) and its registers the other
// axis: the softmax's maximum and sum are then sums over registers and one exchange between half-waves, and the probabilities
// go into the second product from the registers in which the first left them (tessel_tile.h: operand, column_operand).
#include "tessel_block.h"
#include "tessel_tile.h"

namespace tessel {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

// The work of a workgroup.  Tiles are in order of falling work, so that the last ones to start are short.  Workgroups go to the eight
// L2 caches in turn: with heads in eights, each cache sees an eighth of the heads, and those that share keys and values together.
__device__ __forceinline__ void work_of(int heads, int &tile, int &head)
{
    const int b = blockIdx.x;
    if (heads % 8 == 0) {
        const int per = heads / 8, slot = b >> 3;
        tile = slot / per;
        head = (b & 7) * per + slot % per;
    } else {
        tile = b / heads;
        head = b % heads;
    }
}

template <typename T>
__device__ __forceinline__ const T *row_of(const tessel_heads &h, int64_t token, int head)
{
    return (const T *)h.data + token * h.token_stride + head * h.head_stride;
}

__device__ __forceinline__ uint4v load16(const void *p) { return *(const uint4v *)p; }

// the operand of this lane's row straight from memory: columns 16 s + 8 (lane / 32) + 0..7
template <typename T, int W>
__device__ __forceinline__ void fetch_rows(uint4v *v, const T *row, bool valid, int dim)
{
    const int half = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int s = 0; s < W / 16; s++) {
        const int c = 16 * s + 8 * half;
        v[s] = valid && c < dim ? load16(row + c) : uint4v{0, 0, 0, 0};
    }
}

// a 32-column block of a transposed result (lane: one row of the output, registers: its columns) to memory
template <typename T>
__device__ __forceinline__ void put_rows(T *row, const float16v &c, int b, float by, int dim)
{
    const int half = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int d = 32 * b + 8 * i + 4 * half;
        if (d < dim) {
            uint2 w;
            w.x = pack2<T>(c[4 * i] * by, c[4 * i + 1] * by);
            w.y = pack2<T>(c[4 * i + 2] * by, c[4 * i + 3] * by);
            *(uint2 *)(row + d) = w;
        }
    }
}

// zeros for tokens of no sequence
template <typename T>
__device__ void clear_rows(const tessel_heads &h, int begin, int rows, int head, int dim)
{
    const int chunks = dim / 8;
    for (int n = threadIdx.x; n < rows * chunks; n += kThreads)
        *(uint4v *)((T *)row_of<T>(h, begin + n / chunks, head) + 8 * (n % chunks)) = uint4v{0, 0, 0, 0};
}

// Zeros into tiles that will not be filled whole: heads narrower than the tile, or fewer rows than the tiles hold.
template <int N, int W>
__device__ __forceinline__ void clear_tiles(uint4v (*tiles)[64 * W / 8], int rows, int dim)
{
    if (dim == W && rows >= 128) return;
    for (int n = threadIdx.x; n < N * 64 * W / 8; n += kThreads) tiles[0][n] = uint4v{0, 0, 0, 0};
    __syncthreads();
}

template <typename T, int W>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendLaunch l)
{
    __shared__ uint4v buffers[4][64 * W / 8];
    int t, head;
    work_of(l.a.heads, t, head);
    const AttendTile tile = l.tiles[t];
    const int dim = l.a.dim;
    if (tile.length < 0) {
        clear_rows<T>(l.a.o, tile.begin, -tile.length, head, dim);
        for (int n = threadIdx.x; n < -tile.length; n += kThreads) l.a.lse[head * l.tokens + tile.begin + n] = -INFINITY;
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
    const int first = tile.tile * kAttendRows, wfirst = first + 32 * wave, query = wfirst + (lane & 31);
    const int last = min(first + kAttendRows, tile.length);
    const int kv = head / (l.a.heads / l.a.kv_heads);
    const int64_t token = tile.begin + query;
    const bool valid = query < tile.length;

    uint4v q[W / 16];
    fetch_rows<T, W>(q, row_of<T>(l.a.q, token, head), valid, dim);
    float16v o[W / 32] = {};
    float m = -INFINITY, sum = 0;
    const float by = l.a.scale * kLog2e, slack = 8.0f / by;

    const T *kp = row_of<T>(l.a.k, tile.begin, kv), *vp = row_of<T>(l.a.v, tile.begin, kv);
    clear_tiles<4, W>(buffers, last, dim);
    Copy<T, W>::start(buffers[0], kp, l.a.k.token_stride, last, dim);
    Copy<T, W>::start(buffers[1], vp, l.a.v.token_stride, last, dim);
    for (int k0 = 0, turn = 0; k0 < last; k0 += 64, turn ^= 2) {
        const uint4v *keys = buffers[turn], *values = buffers[turn + 1];
        copies_arrive();                                         // (this tile has arrived, and all are done with the one before)
        if (k0 + 64 < last) {
            Copy<T, W>::start(buffers[turn ^ 2], kp + (k0 + 64) * l.a.k.token_stride, l.a.k.token_stride, last - k0 - 64, dim);
            Copy<T, W>::start(buffers[turn ^ 2 | 1], vp + (k0 + 64) * l.a.v.token_stride, l.a.v.token_stride, last - k0 - 64, dim);
        }
        if (k0 > wfirst + 31) continue;
        float16v s[2] = {};
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int n = 0; n < W / 16; n++) s[b] = mma<T>(row_operand<W>(keys, 32 * b, n), q[n], s[b]);
        if (k0 + 63 > wfirst) {
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (k0 + 32 * b + 8 * (i / 4) + 4 * half + i % 4 > query) s[b][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) top = fmaxf(top, s[b][i]);
        top = fmaxf(top, other_half(top));
        // The maximum moves only where it grows by more than a factor of 2^8: until then the probabilities stay below that, which 32 bits and
        // both types hold, and the sums need no scaling.
        if (__any(top > m + slack)) {
            const float next = fmaxf(m, top), shrink = m == next ? 1.0f : __builtin_amdgcn_exp2f((m - next) * by);
            m = next;
            sum *= shrink;
#pragma unroll
            for (int b = 0; b < W / 32; b++) o[b] *= shrink;
        }
        const float at = m == -INFINITY ? 0.0f : m * by;
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                s[b][i] = __builtin_amdgcn_exp2f(s[b][i] * by - at);
                sum += s[b][i];
            }
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const uint4v p = operand<T>(s[n / 2], n % 2);
#pragma unroll
            for (int b = 0; b < W / 32; b++) o[b] = mma<T>(column_operand<W>(values, 16 * n, b), p, o[b]);
        }
    }
    sum += other_half(sum);
    if (!valid) return;
    T *out = (T *)row_of<T>(l.a.o, token, head);
    const float inv = 1.0f / sum;
#pragma unroll
    for (int b = 0; b < W / 32; b++) put_rows<T>(out, o[b], b, inv, dim);
    if (half == 0) l.a.lse[head * l.tokens + token] = m * l.a.scale + logf(sum);
}

// delta_i = sum_d do_i o_i, and in half precision the largest |do| of the launch (by workgroup): the gradients of the scores are scaled by a
// power of two near it before they are rounded, which keeps them in the middle of the type's short range.
//
// The first 128 queries of a sequence take delta_i = sum_j p_ij (do_i . v_j) instead, the same sum from the inputs: o is rounded,
// and where a query sees few keys that error is as large as the one of rounding the gradients of the scores (dq and dk of sequences of 1 to 40 tokens were
// 2.1 times as far from the 64-bit values as the rounding of the results alone puts them, and are 1.4 times now).
template <typename T, int W>
__global__ __launch_bounds__(kThreads) void attend_delta_kernel(AttendLaunch l)
{
    typedef typename Vec8<T>::type V;
    __shared__ float tops[kThreads / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
    const int part = threadIdx.x & 15, dim = l.a.dim;
    float top = 0;
    for (int64_t w = blockIdx.x; w < (int64_t)l.num_tiles * l.a.heads; w += gridDim.x) {
        const AttendTile tile = l.tiles[w / l.a.heads];
        const int head = w % l.a.heads;
        if (tile.length < 0) continue;
        if (tile.tile == 0) {
            const int kv = head / (l.a.heads / l.a.kv_heads), query = 32 * wave + (lane & 31);
            const int64_t token = tile.begin + query;
            const bool valid = query < tile.length;
            uint4v q[W / 16], g[W / 16], k[W / 16], v[W / 16];
            fetch_rows<T, W>(q, row_of<T>(l.a.q, token, head), valid, dim);
            fetch_rows<T, W>(g, row_of<T>(l.a.d_o, token, head), valid, dim);
            const float by = l.a.scale * kLog2e, lse = valid ? l.a.lse[head * l.tokens + token] * kLog2e : 0.0f;
            float sum = 0;
            for (int k0 = 0; k0 <= 32 * wave && k0 < tile.length; k0 += 32) {
                const int key = k0 + (lane & 31);
                fetch_rows<T, W>(k, row_of<T>(l.a.k, tile.begin + key, kv), key < tile.length, dim);
                fetch_rows<T, W>(v, row_of<T>(l.a.v, tile.begin + key, kv), key < tile.length, dim);
                float16v s = {}, d = {};
#pragma unroll
                for (int n = 0; n < W / 16; n++) {
                    s = mma<T>(k[n], q[n], s);
                    d = mma<T>(v[n], g[n], d);
                }
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (k0 + 8 * (i / 4) + 4 * half + i % 4 <= query) sum += __builtin_amdgcn_exp2f(s[i] * by - lse) * d[i];
            }
            sum += other_half(sum);
            if (valid && half == 0) l.delta[head * l.tokens + token] = sum;
            if constexpr (__is_same(T, f16)) {
#pragma unroll
                for (int n = 0; n < W / 16; n++)
#pragma unroll
                    for (int j = 0; j < 8; j++) top = fmaxf(top, fabsf((float)__builtin_bit_cast(V, g[n])[j]));
            }
            continue;
        }
        const int first = tile.tile * kAttendRows, rows = min(kAttendRows, tile.length - first);
        for (int r = threadIdx.x >> 4; r < rows; r += kThreads / 16) {
            const int64_t token = tile.begin + first + r;
            float sum = 0;
            if (8 * part < dim) {
                const V x = __builtin_bit_cast(V, load16(row_of<T>(l.a.o, token, head) + 8 * part));
                const V y = __builtin_bit_cast(V, load16(row_of<T>(l.a.d_o, token, head) + 8 * part));
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    sum += (float)x[j] * (float)y[j];
                    top = fmaxf(top, fabsf((float)y[j]));
                }
            }
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
            if (part == 0) l.delta[head * l.tokens + token] = sum;
        }
    }
    if constexpr (__is_same(T, f16)) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        if (threadIdx.x == 0) l.largest[blockIdx.x] = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    }
}

// the power of two that brings the largest |do| into 1..2 (f16); 1 for bf16, whose range is that of 32 bits
template <typename T>
__device__ __forceinline__ float gradient_scale(const AttendLaunch &l)
{
    if constexpr (__is_same(T, bf16)) return 1.0f;
    float top = 0;
    for (int i = threadIdx.x & 63; i < kAmaxParts; i += 64) top = fmaxf(top, l.largest[i]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (!(top > 0.0f && top < INFINITY)) return 1.0f;
    return __uint_as_float((254u << 23) - (__float_as_uint(top) & 0x7F800000u));
}

template <typename T, int W>
__global__ __launch_bounds__(kThreads, 2) void attend_dq_kernel(AttendLaunch l)
{
    __shared__ uint4v buffers[4][64 * W / 8];
    int t, head;
    work_of(l.a.heads, t, head);
    const AttendTile tile = l.tiles[t];
    const int dim = l.a.dim;
    if (tile.length < 0) {
        clear_rows<T>(l.a.dq, tile.begin, -tile.length, head, dim);
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
    const int first = tile.tile * kAttendRows, wfirst = first + 32 * wave, query = wfirst + (lane & 31);
    const int last = min(first + kAttendRows, tile.length);
    const int kv = head / (l.a.heads / l.a.kv_heads);
    const int64_t token = tile.begin + query;
    const bool valid = query < tile.length;
    const float grow = gradient_scale<T>(l);

    uint4v q[W / 16], g[W / 16];
    fetch_rows<T, W>(q, row_of<T>(l.a.q, token, head), valid, dim);
    fetch_rows<T, W>(g, row_of<T>(l.a.d_o, token, head), valid, dim);
    const float by = l.a.scale * kLog2e;
    const float lse = valid ? l.a.lse[head * l.tokens + token] * kLog2e : 0.0f;
    const float delta = valid ? l.delta[head * l.tokens + token] : 0.0f;
    float16v dq[W / 32] = {};

    const T *kp = row_of<T>(l.a.k, tile.begin, kv), *vp = row_of<T>(l.a.v, tile.begin, kv);
    clear_tiles<4, W>(buffers, last, dim);
    Copy<T, W>::start(buffers[0], kp, l.a.k.token_stride, last, dim);
    Copy<T, W>::start(buffers[1], vp, l.a.v.token_stride, last, dim);
    for (int k0 = 0, turn = 0; k0 < last; k0 += 64, turn ^= 2) {
        const uint4v *keys = buffers[turn], *values = buffers[turn + 1];
        copies_arrive();
        if (k0 + 64 < last) {
            Copy<T, W>::start(buffers[turn ^ 2], kp + (k0 + 64) * l.a.k.token_stride, l.a.k.token_stride, last - k0 - 64, dim);
            Copy<T, W>::start(buffers[turn ^ 2 | 1], vp + (k0 + 64) * l.a.v.token_stride, l.a.v.token_stride, last - k0 - 64, dim);
        }
#pragma unroll
        for (int b = 0; b < 2; b++) {
            if (k0 + 32 * b > wfirst + 31) continue;
            float16v s = {}, d = {};
#pragma unroll
            for (int n = 0; n < W / 16; n++) {
                s = mma<T>(row_operand<W>(keys, 32 * b, n), q[n], s);
                d = mma<T>(row_operand<W>(values, 32 * b, n), g[n], d);
            }
            const bool edge = k0 + 32 * b + 31 > wfirst;
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float p = __builtin_amdgcn_exp2f(s[i] * by - lse);
                s[i] = p * (d[i] - delta) * grow;
                if (edge && k0 + 32 * b + 8 * (i / 4) + 4 * half + i % 4 > query) s[i] = 0.0f;
            }
#pragma unroll
            for (int n = 0; n < 2; n++) {
                const uint4v p = operand<T>(s, n);
#pragma unroll
                for (int c = 0; c < W / 32; c++) dq[c] = mma<T>(column_operand<W>(keys, 32 * b + 16 * n, c), p, dq[c]);
            }
        }
    }
    if (!valid) return;
    T *out = (T *)row_of<T>(l.a.dq, token, head);
    const float back = l.a.scale / grow;
#pragma unroll
    for (int b = 0; b < W / 32; b++) put_rows<T>(out, dq[b], b, back, dim);
}

// Keeps accumulators where they are from one tile to the next (the compiler else moves them to other registers and back in every tile),
// and gives the last product the time that it takes to write them.
template <int W>
__device__ __forceinline__ void keep_sums(float16v *x, float16v *y)
{
    asm volatile("s_nop 15");
#pragma unroll
    for (int c = 0; c < W / 32; c++) asm volatile("" : "+a"(x[c]), "+a"(y[c]));
}

// What a wave of the kernel below does with a tile of 64 queries, its 32 keys against the queries' two blocks of 32.  Four phases of W / 16
// steps of two products each: the scores and dp = do v of block 0, those of block 1, the sums into dv and dk of block 0, those of block 1.  The
// exponentials of block 0 are worked out between the products of the second phase, those of block 1 in the third: with one wave on a
// SIMD (two accumulators of 32 x W leave no room for more) nothing else would run beside the matrix unit.  LDS is read two steps ahead.
template <typename T, int W, bool EDGE>
__device__ __forceinline__ void dkv_tile(const uint4v *queries, const uint4v *grads, const float4v *lses, const float4v *deltas, const uint4v *k,
                                         const uint4v *v, float16v *dk, float16v *dv, float by, float grow, int before)
{
    constexpr int S = W / 16, E = 16 / S;                        // steps a phase, values of a block a step
    const int half = threadIdx.x >> 5 & 1;
    uint4v f[4 * S][2];
    float16v s[2], d[2];
    uint4v p[2][2], e[2][2];
    auto read = [&](int t) {
        if (t >= 4 * S) return;
        const int b = t / S & 1, n = t % S;
        if (t < 2 * S) {
            f[t][0] = row_operand<W>(queries, 32 * b, n);
            f[t][1] = row_operand<W>(grads, 32 * b, n);
        } else {
            const int row = 32 * b + 16 * (n / (W / 32)), c = n % (W / 32);
            f[t][0] = column_operand<W>(queries, row, c);
            f[t][1] = column_operand<W>(grads, row, c);
        }
    };
    // the sums of the first products start from what is taken off them
    auto start = [&](int b) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float4v x = lses[8 * b + 2 * i + half], y = deltas[8 * b + 2 * i + half];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                s[b][4 * i + j] = x[j];
                d[b][4 * i + j] = y[j];
            }
        }
    };
    start(0);
    read(0);
    read(1);
#pragma unroll
    for (int t = 0; t < 4 * S; t++) {
        const int phase = t / S, n = t % S;
        read(t + 2);
        if (t == S - 1) start(1);
        if (phase < 2) {
            s[phase] = mma<T>(f[t][0], k[n], s[phase]);
            d[phase] = mma<T>(f[t][1], v[n], d[phase]);
        } else {
            const int b = phase - 2, c = n % (W / 32), h = n / (W / 32);
            dk[c] = mma<T>(f[t][0], e[b][h], dk[c]);
            dv[c] = mma<T>(f[t][1], p[b][h], dv[c]);
        }
        if (phase == 1 || phase == 2) {
            const int b = phase - 1;
#pragma unroll
            for (int i = n * E; i < (n + 1) * E; i++) {
                float x = __builtin_amdgcn_exp2f(s[b][i] * by);
                if (EDGE && 32 * b + 8 * (i / 4) + i % 4 < before) x = 0.0f;
                d[b][i] *= __is_same(T, f16) ? x * grow : x;
                s[b][i] = x;
                if (i % 8 == 7) {
                    p[b][i / 8] = operand<T>(s[b], i / 8);
                    e[b][i / 8] = operand<T>(d[b], i / 8);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    keep_sums<W>(dk, dv);
}

template <typename T, int W>
__global__ __launch_bounds__(kThreads, 1) void attend_dkv_kernel(AttendLaunch l)
{
    __shared__ uint4v buffers[4][64 * W / 8];
    __shared__ float4v numbers[2][2][16];                        // - log-sum / scale and - delta of a tile's queries
    int t, kv;
    work_of(l.a.kv_heads, t, kv);
    const AttendTile tile = l.tiles[t];
    const int dim = l.a.dim;
    if (tile.length < 0) {
        clear_rows<T>(l.a.dk, tile.begin, -tile.length, kv, dim);
        clear_rows<T>(l.a.dv, tile.begin, -tile.length, kv, dim);
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
    // (the tile with the most keys before it has the fewest queries behind it: the order of falling work is turned round)
    const int first = (tile.tiles - 1 - tile.tile) * kAttendRows, key = first + 32 * wave + (lane & 31);
    const int64_t token = tile.begin + key;
    const bool valid = key < tile.length;
    const int shared = l.a.heads / l.a.kv_heads;
    const float grow = gradient_scale<T>(l);

    uint4v k[W / 16], v[W / 16];
    fetch_rows<T, W>(k, row_of<T>(l.a.k, token, kv), valid, dim);
    fetch_rows<T, W>(v, row_of<T>(l.a.v, token, kv), valid, dim);
    const float by = l.a.scale * kLog2e;
    float16v dk[W / 32] = {}, dv[W / 32] = {};

    // the tiles of all heads that share these keys, one behind the other
    const int tiles = (tile.length - first + 63) / 64, edges = min(tiles, kAttendRows / 64), all = tiles * shared;
    float number = 0;                                            // (on its way to LDS, one tile ahead)
    auto fetch = [&](int n) {
        const int head = kv * shared + n / tiles, q0 = first + n % tiles * 64, rows = tile.length - q0;
        uint4v (*to)[64 * W / 8] = buffers + 2 * (n & 1);
        Copy<T, W>::start(to[0], row_of<T>(l.a.q, tile.begin + q0, head), l.a.q.token_stride, rows, dim);
        Copy<T, W>::start(to[1], row_of<T>(l.a.d_o, tile.begin + q0, head), l.a.d_o.token_stride, rows, dim);
        if (threadIdx.x < 128) {
            const int r = threadIdx.x & 63;
            const int64_t at = head * l.tokens + tile.begin + q0 + r;
            // (queries behind the sequence's end: a probability of nought)
            if (threadIdx.x < 64) number = r < rows ? -l.a.lse[at] / l.a.scale : -INFINITY;
            else number = r < rows ? -l.delta[at] : 0.0f;
        }
    };
    auto next = [&](int n) {
        if (threadIdx.x < 128) ((float *)numbers[n & 1])[threadIdx.x] = number;
        copies_arrive();                                         // (tile n has arrived, and all are done with the one before)
        if (n + 1 < all) fetch(n + 1);
    };
    clear_tiles<4, W>(buffers, tile.length - first, dim);
    fetch(0);
    for (int n = 0; n < all;) {
        for (int i = 0; i < edges; i++, n++) {
            next(n);
            dkv_tile<T, W, true>(buffers[2 * (n & 1)], buffers[2 * (n & 1) + 1], numbers[n & 1][0], numbers[n & 1][1], k, v, dk, dv, by, grow,
                                 32 * wave + (lane & 31) - 64 * i - 4 * half);
        }
        for (int i = edges; i < tiles; i++, n++) {
            next(n);
            dkv_tile<T, W, false>(buffers[2 * (n & 1)], buffers[2 * (n & 1) + 1], numbers[n & 1][0], numbers[n & 1][1], k, v, dk, dv, by, grow, 0);
        }
    }
    if (!valid) return;
    const float back = l.a.scale / grow;
    T *dkp = (T *)row_of<T>(l.a.dk, token, kv), *dvp = (T *)row_of<T>(l.a.dv, token, kv);
#pragma unroll
    for (int b = 0; b < W / 32; b++) {
        put_rows<T>(dkp, dk[b], b, back, dim);
        put_rows<T>(dvp, dv[b], b, 1.0f, dim);
    }
}

static int launch(const void *kernel, int64_t blocks, const AttendLaunch &l, void *stream)
{
    AttendLaunch copy = l;
    void *args[] = {&copy};
    const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)blocks), dim3(kThreads), args, 0, (hipStream_t)stream);
    if (e != hipSuccess) (void)hipGetLastError();
    return (int)e;
}

// heads of up to 64 run in tiles 64 wide: half the work of 128
#define ATTEND_KERNEL(name) (l.a.type == TESSEL_BF16 ? (l.a.dim <= 64 ? (const void *)name<bf16, 64> : (const void *)name<bf16, 128>) \
                                                     : (l.a.dim <= 64 ? (const void *)name<f16, 64> : (const void *)name<f16, 128>))

int launch_attend(const AttendLaunch &l, void *stream)
{
    return launch(ATTEND_KERNEL(attend_kernel), (int64_t)l.num_tiles * l.a.heads, l, stream);
}

int launch_attend_backward(const AttendLaunch &l, void *stream)
{
    int e = launch(ATTEND_KERNEL(attend_delta_kernel), kAmaxParts, l, stream);
    if (e == 0) e = launch(ATTEND_KERNEL(attend_dkv_kernel), (int64_t)l.num_tiles * l.a.kv_heads, l, stream);
    if (e == 0) e = launch(ATTEND_KERNEL(attend_dq_kernel), (int64_t)l.num_tiles * l.a.heads, l, stream);
    return e;
}

}  // namespace tessel
