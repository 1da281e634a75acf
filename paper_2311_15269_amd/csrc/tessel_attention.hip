// Causal attention over packed sequences with grouped heads, forward and backward (formulas: include/tessel_block_ops.h).
//
// A workgroup of four waves takes 128 queries of one head (or, for the gradients of k and v, 128 keys of a key-value head), 32 a wave.  All
// products are 32 x 32 x 16 matrix instructions, arranged so that a lane of the score tile holds ONE query (key) and its registers the other
// axis: the softmax's maximum and sum are then sums over registers and one exchange between half-waves, and the probabilities
// go into the second product from the registers in which the first left them (tessel_tile.h: operand, read_columns).  Tiles of 64 rows
// come from memory straight to LDS, the next ones while these are worked on.
//
// Bounds.  A wave's product of 32 x 32 x 128 keeps a matrix unit busy for 256 clocks and reads one operand of 8 KB from LDS, which takes 256
// clocks to serve all four SIMDs: both are as busy as each other, and the softmax's instructions (16 exponentials a lane for two products) are
// some 40 % of that beside them.  Two waves on a SIMD fill each other's gaps, with what 256 registers a lane hold: 32 queries with all of
// their sums.  Under this load the card lowers its clock (1.6 - 2.0 GHz); a large library product reaches 1260 TF/s in that state.
#include <algorithm>

#include "tessel_block.h"
#include "tessel_tile.h"

namespace tessel {

constexpr int kThreads = kAttendThreads;
constexpr int kAhead = 4;        // operands that are read from LDS ahead of their products
constexpr float kLog2e = 1.4426950408889634f;

// The work of a workgroup.  Tiles are in order of falling work, so that the last ones to start are short.  Workgroups go to the eight
// L2 caches in turn: with heads (times splits) in eights, each cache sees an eighth of the heads, and those that share keys and values together.
__device__ __forceinline__ void work_of(int heads, int splits, int &tile, int &head, int &split)
{
    const int b = blockIdx.x, all = heads * splits;
    int which;
    if (all % 8 == 0) {
        const int per = all / 8, slot = b >> 3;
        tile = slot / per;
        which = (b & 7) * per + slot % per;
    } else {
        tile = b / all;
        which = b % all;
    }
    head = which / splits;
    split = which % splits;
}

// The steps of split `split` of a tile with `all` of them, first .. end - 1: shares as even as whole steps allow.  (With fewer steps than splits the
// first splits have one each, the others none.)
__device__ __forceinline__ void share_of(int all, int splits, int split, int &first, int &end)
{
    const int sharing = min(all, splits);
    first = split < sharing ? (int)((int64_t)all * split / sharing) : all;
    end = split < sharing ? (int)((int64_t)all * (split + 1) / sharing) : all;
}

// this wave's number in its workgroup, in a scalar register: what is compared with it is one branch for the wave
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

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

// the same in 32 bits, into a split's part
__device__ __forceinline__ void put_part(float *row, const float16v &c, int b, float by, int dim)
{
    const int half = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int d = 32 * b + 8 * i + 4 * half;
        if (d < dim) *(float4v *)(row + d) = float4v{c[4 * i] * by, c[4 * i + 1] * by, c[4 * i + 2] * by, c[4 * i + 3] * by};
    }
}

// zeros for tokens of no sequence
template <typename T>
__device__ void clear_rows(const tessel_heads &h, int begin, int rows, int head, int dim)
{
    const int chunks = dim / 8;
    for (int n = threadIdx.x; n < rows * chunks; n += blockDim.x)
        *(uint4v *)((T *)row_of<T>(h, begin + n / chunks, head) + 8 * (n % chunks)) = uint4v{0, 0, 0, 0};
}

// Zeros into tiles that will not be filled whole: heads narrower than the tile, or fewer rows than the tiles hold.
template <int N, int W, int THREADS = kThreads>
__device__ __forceinline__ void clear_tiles(uint4v (*tiles)[64 * W / 8], int rows, int dim)
{
    if (dim == W && rows >= 128) return;
    for (int n = threadIdx.x; n < N * 64 * W / 8; n += THREADS) tiles[0][n] = uint4v{0, 0, 0, 0};
    __syncthreads();
}

// the sign bits of those halves of a word that hold an infinity or NaN
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x)
{
    return __is_same(T, bf16) ? ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u : ((x & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
}

// A query's probability of a key behind it is nought, but nought times infinity or NaN is not.  Where sixteen rows of values `f`, from row
// `row` of the tile on, hold any: they are taken out of the product, and added for those queries that see them.
template <typename T, int W>
__device__ __forceinline__ void part_with_later(uint4v (&f)[W / 32], float16v *o, const lds_tile *values, int row, int seen)
{
    uint32_t any = 0;
#pragma unroll
    for (int b = 0; b < W / 32; b++)
#pragma unroll
        for (int j = 0; j < 4; j++) any |= not_finite<T>(f[b][j]);
    if (!__any(any != 0u)) return;
#pragma unroll
    for (int b = 0; b < W / 32; b++)
#pragma unroll
        for (int j = 0; j < 4; j++) f[b][j] &= ~((not_finite<T>(f[b][j]) >> 15) * 0xFFFFu);
    const int half = threadIdx.x >> 5 & 1;
#pragma unroll 1
    for (int r = row; r < row + 16 && r <= seen; r++) {
#pragma unroll
        for (int b = 0; b < W / 32; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                typedef T V __attribute__((ext_vector_type(8)));
                const V v = __builtin_bit_cast(V, (uint4v)values[chunk_at<W>(r, 4 * b + i)]);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float x = half ? (float)v[4 + j] : (float)v[j];
                    o[b][4 * i + j] += fabsf(x) < INFINITY ? 0.0f : x;
                }
                __builtin_amdgcn_sched_barrier(0);               // (one value after the other: this is rare, and its registers count for all)
            }
    }
}

// Keys and values once over, with the largest score and the sum of a query's exponentials kept as it goes.  One prompt of 16384 tokens, 32
// heads of 128 on 8 of keys: 2.13 ms, 1030 TF/s; documents of 1 to 3001 tokens, 8192 in all, 32 heads: 179 us, 760 TF/s (a workgroup has 17 steps of 64
// keys on average where the prompt's has 129, so that its first reads, one behind the other, and its end weigh more, and a tenth of its scores
// is masked); 58 tokens in three sequences: 5.6 us.
template <typename T, int W>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendLaunch l)
{
    __shared__ __attribute__((aligned(256))) uint4v buffers[4][64 * W / 8];
    int t, head, split;
    work_of(l.a.heads, l.splits, t, head, split);
    const AttendTile tile = l.tiles[t];
    const int dim = l.a.dim;
    if (tile.length < 0) {
        if (split) return;
        clear_rows<T>(l.a.o, tile.begin, -tile.length, head, dim);
        for (int n = threadIdx.x; n < -tile.length; n += kThreads) l.a.lse[head * l.tokens + tile.begin + n] = -INFINITY;
        return;
    }
    const int wave = wave_number(), lane = threadIdx.x & 63, half = lane >> 5;
    const int first = tile.tile * kAttendRows, wfirst = first + 32 * wave, query = wfirst + (lane & 31);
    const int last = min(first + kAttendRows, tile.length);
    int from, to;
    share_of((last + 63) / 64, l.splits, split, from, to);
    if (from == to) return;
    from *= 64;
    to = min(64 * to, last);
    const int kv = head / (l.a.heads / l.a.kv_heads);
    const int64_t token = tile.begin + query;
    const bool valid = query < tile.length;

    uint4v q[W / 16];
    fetch_rows<T, W>(q, row_of<T>(l.a.q, token, head), valid, dim);
    float16v o[W / 32] = {};
    float m = -INFINITY, sum = 0;
    const float by = l.a.scale * kLog2e, slack = 8.0f / by;

    const T *kp = row_of<T>(l.a.k, tile.begin, kv), *vp = row_of<T>(l.a.v, tile.begin, kv);
    Reader<W> at;
    clear_tiles<4, W>(buffers, to - from, dim);
    Copy<T, W, kThreads>::start(buffers[0], kp + from * l.a.k.token_stride, l.a.k.token_stride, to - from, dim);
    Copy<T, W, kThreads>::start(buffers[1], vp + from * l.a.v.token_stride, l.a.v.token_stride, to - from, dim);
    for (int k0 = from, turn = 0; k0 < to; k0 += 64, turn ^= 2) {
        const lds_tile *keys = (const lds_tile *)buffers[turn], *values = (const lds_tile *)buffers[turn + 1];
        copies_arrive();                                         // (this tile has arrived, and all are done with the one before)
        if (k0 + 64 < to) {
            Copy<T, W, kThreads>::start(buffers[turn ^ 2], kp + (k0 + 64) * l.a.k.token_stride, l.a.k.token_stride, to - k0 - 64, dim);
            Copy<T, W, kThreads>::start(buffers[turn ^ 2 | 1], vp + (k0 + 64) * l.a.v.token_stride, l.a.v.token_stride, to - k0 - 64, dim);
        }
        if (k0 > wfirst + 31) continue;
        // (LDS is read a few products ahead: the compiler would wait for each operand right behind its read)
        float16v s[2] = {};
        uint4v f[W / 8];
#pragma unroll
        for (int t = 0; t < kAhead; t++) f[t] = at.rows(keys, 32 * (t % 2), t / 2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < W / 8; t++) {
            if (t + kAhead < W / 8) f[t + kAhead] = at.rows(keys, 32 * (t % 2), (t + kAhead) / 2);
            s[t % 2] = mma<T>(f[t], q[t / 2], s[t % 2]);
            __builtin_amdgcn_sched_barrier(0);
        }
        const bool edge = k0 + 63 > wfirst;
        if (edge) {
            const int seen = query - k0 - 4 * half;
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (32 * b + 8 * (i / 4) + i % 4 > seen) s[b][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) top = fmaxf(top, s[b][i]);
        top = max_of_halves(top);
        // The maximum moves only where it grows by more than a factor of 2^8: until then the probabilities stay below that, which 32 bits and
        // both types hold, and the sums need no scaling.
        if (__any(top > m + slack)) {
            const float next = fmaxf(m, top), shrink = m == next ? 1.0f : __builtin_amdgcn_exp2f((m - next) * by);
            m = next;
            sum *= shrink;
#pragma unroll
            for (int b = 0; b < W / 32; b++) o[b] *= shrink;
        }
        const float off = m == -INFINITY ? 0.0f : m * by;
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                s[b][i] = __builtin_amdgcn_exp2f(s[b][i] * by - off);
                sum += s[b][i];
            }
        uint32_t va[W / 16];
        column_addresses<W>(va, values, at);
        unrolled<4>([&](auto c) {
            constexpr int n = decltype(c)::value;
            const uint4v p = operand<T>(s[n / 2], n % 2);
            uint4v f[W / 32];
            read_columns<32 * n * W>(f, va);
            if (edge) part_with_later<T, W>(f, o, values, 16 * n, query - k0);
#pragma unroll
            for (int b = 0; b < W / 32; b++) o[b] = mma<T>(f[b], p, o[b]);
        });
    }
    sum = sum_of_halves(sum);
    if (!valid) return;
    if (l.splits > 1) {
        const int64_t row = ((int64_t)split * l.a.heads + head) * l.tokens + token;
#pragma unroll
        for (int b = 0; b < W / 32; b++) put_part(l.parts + row * dim, o[b], b, 1.0f, dim);
        if (half == 0) {
            l.tops[2 * row] = m;
            l.tops[2 * row + 1] = sum;
        }
        return;
    }
    T *out = (T *)row_of<T>(l.a.o, token, head);
    const float inv = 1.0f / sum;
#pragma unroll
    for (int b = 0; b < W / 32; b++) put_rows<T>(out, o[b], b, inv, dim);
    if (half == 0) l.a.lse[head * l.tokens + token] = m * l.a.scale + logf(sum);
}

// Joins the parts of the forward pass (FORWARD: sums of exponentials that each go by their own largest score) or adds up those of gradients,
// in the order of the splits.  Eight rows a workgroup, 32 lanes of four columns each.  blockIdx.y: of the two arrays that a part of dk and
// dv holds one behind the other; steps_by: heads on a key, `turned`: tiles of keys (see attend_dkv_kernel).
template <typename T, bool FORWARD>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendLaunch l, tessel_heads first_out, tessel_heads second_out, int heads, int steps_by, bool turned)
{
    constexpr int kGroups = kAttendRows / kJoinRows;
    const int group = blockIdx.x % kGroups, head = blockIdx.x / kGroups % heads;
    const AttendTile tile = l.tiles[blockIdx.x / kGroups / heads];
    if (tile.length < 0) return;
    const int col = 4 * (threadIdx.x & 31), dim = l.a.dim;
    const int first = (turned ? tile.tiles - 1 - tile.tile : tile.tile) * kAttendRows, r = first + group * kJoinRows + (threadIdx.x >> 5);
    if (r >= tile.length) return;
    const int steps = turned ? (tile.length - first + 63) / 64 * steps_by : (min(first + kAttendRows, tile.length) + 63) / 64;
    const int parts = min(steps, l.splits);
    const int64_t token = tile.begin + r, row = ((int64_t)blockIdx.y * heads + head) * l.tokens + token, next = (int64_t)gridDim.y * heads * l.tokens;
    float top = -INFINITY, total = 0;
    if constexpr (FORWARD)
#pragma unroll 4
        for (int s = 0; s < parts; s++) top = fmaxf(top, l.tops[2 * (row + s * next)]);
    float4v sum = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < parts; s++) {
        float by = 1.0f;
        if constexpr (FORWARD) {
            const float2 t = *(const float2 *)(l.tops + 2 * (row + s * next));
            by = t.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((t.x - top) * (l.a.scale * kLog2e));
            total += by * t.y;
        }
        if (col < dim) sum += *(const float4v *)(l.parts + (row + s * next) * dim + col) * by;
    }
    if (col < dim) {
        const float by = FORWARD ? 1.0f / total : 1.0f;
        uint2 w;
        w.x = pack2<T>(sum[0] * by, sum[1] * by);
        w.y = pack2<T>(sum[2] * by, sum[3] * by);
        *(uint2 *)((T *)row_of<T>(blockIdx.y ? second_out : first_out, token, head) + col) = w;
    }
    if (FORWARD && col == 0) l.a.lse[head * l.tokens + token] = top * l.a.scale + logf(total);
}

// In half precision the gradients of the scores are rounded in units of their own, 1 / grow, and what is summed from them with it: a lane of either kernel
// below has the scores of one query (key), so it keeps the unit that its largest gradient so far needs.  `top`: the largest of a block of 32 scores.
// Where it would pass 2^15, the unit goes to where it is 2^8: what is 2^-22 of the largest still has all of the type's bits.  The first
// block sets it, as grow starts where nothing fits.  (The sizes of do and v together say nothing of do . v - delta, let alone of one key's.)
template <int N>
__device__ __forceinline__ void fit(float top, float &grow, float16v *sums)
{
    top = max_of_halves(top);
    const bool over = top * grow > 0x1p15f && top < INFINITY;
    if (!__any(over)) return;
    const float next = over ? __uint_as_float((262u << 23) - (__float_as_uint(top) & 0x7F800000u)) : grow, by = next / grow;
    grow = next;
#pragma unroll
    for (int b = 0; b < N; b++) sums[b] *= by;
}
template <typename T>
__device__ __forceinline__ constexpr float first_grow() { return __is_same(T, f16) ? 0x1p126f : 1.0f; }

// The gradient of q: three products (scores, do v, and their gradients times k), one operand from LDS for each.  The documents above: 246 us, 830
// TF/s.  (It and the kernel of dk and dv both compute the scores, seven products instead of five: one kernel for all three gradients would add
// to dq from many workgroups, in no fixed order.)  Also, for the kernel behind it, delta_i = sum_d do_i o_i.
//
// The first 128 queries of a sequence take delta_i = sum_j p_ij (do_i . v_j) instead, the same sum from the inputs: o is rounded,
// and where a query sees few keys that error is as large as the one of rounding the gradients of the scores.  (dq and dk of sequences of 1, 17
// and 40 tokens in half precision are 2.9e-4 off the 64-bit values with it, 3.4e-4 without; rounding the results alone: 2.1e-4.)
template <typename T, int W>
__global__ __launch_bounds__(kThreads, 2) void attend_dq_kernel(AttendLaunch l)
{
    __shared__ __attribute__((aligned(256))) uint4v buffers[4][64 * W / 8];
    int t, head, split;
    work_of(l.a.heads, l.splits, t, head, split);
    const AttendTile tile = l.tiles[t];
    const int dim = l.a.dim;
    if (tile.length < 0) {
        if (split) return;
        clear_rows<T>(l.a.dq, tile.begin, -tile.length, head, dim);
        return;
    }
    const int wave = wave_number(), lane = threadIdx.x & 63, half = lane >> 5;
    const int first = tile.tile * kAttendRows, wfirst = first + 32 * wave, query = wfirst + (lane & 31);
    const int last = min(first + kAttendRows, tile.length);
    int from, to;
    share_of((last + 63) / 64, l.splits, split, from, to);
    if (from == to) return;
    from *= 64;
    to = min(64 * to, last);
    const int kv = head / (l.a.heads / l.a.kv_heads);
    const int64_t token = tile.begin + query;
    const bool valid = query < tile.length;

    typedef typename Vec8<T>::type V;
    uint4v q[W / 16], g[W / 16];
    fetch_rows<T, W>(q, row_of<T>(l.a.q, token, head), valid, dim);
    fetch_rows<T, W>(g, row_of<T>(l.a.d_o, token, head), valid, dim);
    const float by = l.a.scale * kLog2e;
    const float lse = valid ? l.a.lse[head * l.tokens + token] * kLog2e : 0.0f;
    float delta = 0;
    if (tile.tile == 0) {
        uint4v k[W / 16], v[W / 16];
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
                if (k0 + 8 * (i / 4) + 4 * half + i % 4 <= query) delta += __builtin_amdgcn_exp2f(s[i] * by - lse) * d[i];
        }
    } else {
        uint4v o[W / 16];
        fetch_rows<T, W>(o, row_of<T>(l.a.o, token, head), valid, dim);
#pragma unroll
        for (int n = 0; n < W / 16; n++)
#pragma unroll
            for (int j = 0; j < 8; j++) delta += (float)__builtin_bit_cast(V, o[n])[j] * (float)__builtin_bit_cast(V, g[n])[j];
    }
    delta = sum_of_halves(delta);
    if (valid && half == 0 && to == last) l.delta[head * l.tokens + token] = delta;
    float16v dq[W / 32] = {};
    float grow = first_grow<T>();

    const T *kp = row_of<T>(l.a.k, tile.begin, kv), *vp = row_of<T>(l.a.v, tile.begin, kv);
    Reader<W> at;
    clear_tiles<4, W>(buffers, to - from, dim);
    Copy<T, W, kThreads>::start(buffers[0], kp + from * l.a.k.token_stride, l.a.k.token_stride, to - from, dim);
    Copy<T, W, kThreads>::start(buffers[1], vp + from * l.a.v.token_stride, l.a.v.token_stride, to - from, dim);
    for (int k0 = from, turn = 0; k0 < to; k0 += 64, turn ^= 2) {
        const lds_tile *keys = (const lds_tile *)buffers[turn], *values = (const lds_tile *)buffers[turn + 1];
        copies_arrive();
        if (k0 + 64 < to) {
            Copy<T, W, kThreads>::start(buffers[turn ^ 2], kp + (k0 + 64) * l.a.k.token_stride, l.a.k.token_stride, to - k0 - 64, dim);
            Copy<T, W, kThreads>::start(buffers[turn ^ 2 | 1], vp + (k0 + 64) * l.a.v.token_stride, l.a.v.token_stride, to - k0 - 64, dim);
        }
        uint32_t ka[W / 16];
        column_addresses<W>(ka, keys, at);
        unrolled<2>([&](auto block) {
            constexpr int b = decltype(block)::value;
            if (k0 + 32 * b > wfirst + 31) return;
            float16v s = {}, d = {};
            uint4v x[W / 16], y[W / 16];
#pragma unroll
            for (int n = 0; n < kAhead / 2; n++) {
                x[n] = at.rows(keys, 32 * b, n);
                y[n] = at.rows(values, 32 * b, n);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < W / 16; n++) {
                if (n + kAhead / 2 < W / 16) {
                    x[n + kAhead / 2] = at.rows(keys, 32 * b, n + kAhead / 2);
                    y[n + kAhead / 2] = at.rows(values, 32 * b, n + kAhead / 2);
                }
                s = mma<T>(x[n], q[n], s);
                d = mma<T>(y[n], g[n], d);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float p = __builtin_amdgcn_exp2f(s[i] * by - lse);
                s[i] = p * (d[i] - delta);
            }
            if (k0 + 32 * b + 31 > wfirst) {
                const int seen = query - k0 - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (32 * b + 8 * (i / 4) + i % 4 > seen) s[i] = 0.0f;
            }
            if constexpr (__is_same(T, f16)) {
                float top = 0;
#pragma unroll
                for (int i = 0; i < 16; i++) top = fmaxf(top, fabsf(s[i]));
                fit<W / 32>(top, grow, dq);
                s *= grow;
            }
            unrolled<2>([&](auto h) {
                constexpr int n = decltype(h)::value;
                const uint4v p = operand<T>(s, n);
                uint4v f[W / 32];
                read_columns<32 * (2 * b + n) * W>(f, ka);
#pragma unroll
                for (int c = 0; c < W / 32; c++) dq[c] = mma<T>(f[c], p, dq[c]);
            });
        });
    }
    if (!valid) return;
    T *out = (T *)row_of<T>(l.a.dq, token, head);
    const float back = l.a.scale / grow;
    if (l.splits > 1) {
        float *part = l.parts + (((int64_t)split * l.a.heads + head) * l.tokens + token) * dim;
#pragma unroll
        for (int b = 0; b < W / 32; b++) put_part(part, dq[b], b, back, dim);
        return;
    }
#pragma unroll
    for (int b = 0; b < W / 32; b++) put_rows<T>(out, dq[b], b, back, dim);
}

// In half precision the probabilities for dv are held 2^12 times as large: the type's normal numbers end at 2^-14, and a query that sees 2^16 keys alike
// gives each 2^-16 (rounded as it is, dv of the last of 200000 tokens is off by 3.5e-3 of its norm).  A probability is 1 at most.
constexpr float kRaise = 12.0f, kLower = 0x1p-12f;

// What a wave of the kernel below does with a block of 32 queries and its 32 keys.  LDS is read one step ahead of the products.  `copy` starts
// the copies of the next tile: behind the first products, as the compiler lets no read of LDS that it places itself pass a copy.
template <typename T, int W, bool EDGE, typename F>
__device__ __forceinline__ void dkv_block(const lds_tile *queries, const lds_tile *grads, int row, Reader<W> at, const float4v *lses, const float4v *deltas, const uint4v *k,
                                          const uint4v *values, float16v *dk, float16v *dv, float by, float &grow, int before, F &&copy)
{
    constexpr int S = W / 16;                                    // steps a phase, two products each
    const int half = threadIdx.x >> 5 & 1;
    at.hold();
    uint4v f[S][2], v[S];
    float16v s, d;
    uint4v p[2], e[2];
    auto read = [&](int t) {
        f[t][0] = at.rows(queries, row, t);
        f[t][1] = at.rows(grads, row, t);
        v[t] = values[64 * t];
    };
    read(0);
    // the sums of the first products start from what is taken off them
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float4v x = lses[row / 4 + 2 * i + half], y = deltas[row / 4 + 2 * i + half];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            s[4 * i + j] = x[j];
            d[4 * i + j] = y[j];
        }
    }
    read(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < S; t++) {
        if (t + 2 < S) read(t + 2);
        s = mma<T>(f[t][0], k[t], s);
        d = mma<T>(f[t][1], v[t], d);
        __builtin_amdgcn_sched_barrier(0);
    }
    copy();
#pragma unroll
    for (int i = 0; i < 16; i++) {
        float x = __builtin_amdgcn_exp2f(__is_same(T, f16) ? s[i] * by + kRaise : s[i] * by);
        if (EDGE && 8 * (i / 4) + i % 4 < before) x = 0.0f;
        d[i] *= x;
        s[i] = x;
    }
    if constexpr (__is_same(T, f16)) {
        float top = 0;
#pragma unroll
        for (int i = 0; i < 16; i++) top = fmaxf(top, fabsf(d[i]));
        fit<W / 32>(top, grow, dk);
        d *= grow;
    }
#pragma unroll
    for (int h = 0; h < 2; h++) {
        p[h] = operand<T>(s, h);
        e[h] = operand<T>(d, h);
    }
    __builtin_amdgcn_sched_barrier(0);
    unrolled<2>([&](auto c) {
        constexpr int h = decltype(c)::value;
        uint32_t qa[W / 16];
        uint4v x[W / 32];
        column_addresses<W>(qa, grads + row * W / 8, at);
        read_columns<32 * h * W>(x, qa);
#pragma unroll
        for (int b = 0; b < W / 32; b++) dv[b] = mma<T>(x[b], p[h], dv[b]);
        column_addresses<W>(qa, queries + row * W / 8, at);
        read_columns<32 * h * W>(x, qa);
#pragma unroll
        for (int b = 0; b < W / 32; b++) dk[b] = mma<T>(x[b], e[h], dk[b]);
    });
}

// The gradients of k and v: four products, and five operands from LDS for them, as registers hold the sums of both (128), the keys' operands (32) and
// the scores' (32), but not the values'.  The documents above take 389 us, 710 TF/s.  LDS, 2,560 clocks for 2,048 of products, leaves 1000 TF/s of the
// 1260; what is lost beside that is a wait in every tile: its log-sums and deltas are read behind the copies of the same tile and used at
// once, and as reads come back in order, two of the eight waves stand there until all of those copies have arrived.  (One wave on a SIMD with twice the
// registers: 440 us; queries in tiles of 32 for two workgroups on a compute unit: the same.)
//
// Eight waves: the first four take the tile's first 32 queries, the others the last 32, each 32 of the workgroup's 128 keys; two
// waves on a SIMD, so that one's exponentials run beside the other's products.  At the end the second four hand their sums to the first.
template <typename T, int W>
__global__ __launch_bounds__(kDkvThreads, 2) void attend_dkv_kernel(AttendLaunch l)
{
    __shared__ __attribute__((aligned(256))) uint4v buffers[4][64 * W / 8], values[128 * W / 8];
    __shared__ float4v numbers[2][2][16];                        // - log-sum / scale and - delta of a tile's queries
    int t, kv, split;
    work_of(l.a.kv_heads, l.splits, t, kv, split);
    const AttendTile tile = l.tiles[t];
    const int dim = l.a.dim;
    if (tile.length < 0) {
        if (split) return;
        clear_rows<T>(l.a.dk, tile.begin, -tile.length, kv, dim);
        clear_rows<T>(l.a.dv, tile.begin, -tile.length, kv, dim);
        return;
    }
    const int wave = threadIdx.x >> 6 & 3, row = threadIdx.x >> 8 << 5, lane = threadIdx.x & 63, half = lane >> 5;
    // (the tile with the most keys before it has the fewest queries behind it: the order of falling work is turned round)
    const int first = (tile.tiles - 1 - tile.tile) * kAttendRows, key = first + 32 * wave + (lane & 31);
    const int64_t token = tile.begin + key;
    const bool valid = key < tile.length;
    const int shared = l.a.heads / l.a.kv_heads;
    // the tiles of all heads that share these keys, one behind the other, and of those this split's share
    const int tiles = (tile.length - first + 63) / 64;
    int from, to;
    share_of(tiles * shared, l.splits, split, from, to);
    if (from == to) return;

    uint4v k[W / 16], v[W / 16];
    fetch_rows<T, W>(k, row_of<T>(l.a.k, token, kv), valid, dim);
    fetch_rows<T, W>(v, row_of<T>(l.a.v, token, kv), valid, dim);
    uint4v *const mine = values + wave * (W / 16 * 64) + lane;   // (registers hold the keys' operands; the values' lie in LDS as the lanes need them)
#pragma unroll
    for (int n = 0; n < W / 16; n++) mine[64 * n] = v[n];        // (both waves of these keys: the same)
    const float by = l.a.scale * kLog2e;
    float16v dk[W / 32] = {}, dv[W / 32] = {};

    float number = 0;                                            // (on its way to LDS, one tile ahead)
    auto fetch = [&](int n) {
        const int head = kv * shared + n / tiles, q0 = first + n % tiles * 64, rows = tile.length - q0;
        uint4v (*to)[64 * W / 8] = buffers + 2 * (n & 1);
        Copy<T, W, kDkvThreads>::start(to[0], row_of<T>(l.a.q, tile.begin + q0, head), l.a.q.token_stride, rows, dim);
        Copy<T, W, kDkvThreads>::start(to[1], row_of<T>(l.a.d_o, tile.begin + q0, head), l.a.d_o.token_stride, rows, dim);
        if (threadIdx.x < 128) {
            const int r = threadIdx.x & 63;
            const int64_t at = head * l.tokens + tile.begin + q0 + r;
            // (queries behind the sequence's end: a probability of nought)
            if (threadIdx.x < 64) number = r < rows ? -l.a.lse[at] / l.a.scale : -INFINITY;
            else number = r < rows ? -l.delta[at] : 0.0f;
        }
    };
    float grow = first_grow<T>();
    const Reader<W> at;
    // (a head's last tile may be short: where it comes first or second, nothing has filled the rows behind it yet)
    clear_tiles<4, W, kDkvThreads>(buffers, from % tiles + 2 >= tiles ? 0 : 128, dim);
    fetch(from);
    for (int n = from; n < to; n++) {
        if (threadIdx.x < 128) ((float *)numbers[n & 1])[threadIdx.x] = number;
        copies_arrive();                                         // (tile n has arrived, and all are done with the one before)
        auto copy = [&]() {
            if (n + 1 < to) fetch(n + 1);
        };
        const lds_tile *queries = (const lds_tile *)buffers[2 * (n & 1)], *grads = (const lds_tile *)buffers[2 * (n & 1) + 1];
        const float4v *lses = numbers[n & 1][0], *deltas = numbers[n & 1][1];
        const int before = 32 * wave - n % tiles * 64 - row;     // (this block's queries of which the wave's first key is ahead)
        if (before > 31) copy();
        else if (before > -32) dkv_block<T, W, true>(queries, grads, row, at, lses, deltas, k, mine, dk, dv, by, grow, before + (lane & 31) - 4 * half, copy);
        else dkv_block<T, W, false>(queries, grads, row, at, lses, deltas, k, mine, dk, dv, by, grow, 0, copy);
    }
    float4v *sums = (float4v *)buffers + wave * (W / 32 * 4 * 64) + lane;
    constexpr float lower = __is_same(T, f16) ? kLower : 1.0f;
    if constexpr (__is_same(T, f16)) {
#pragma unroll
        for (int b = 0; b < W / 32; b++) dk[b] *= 1.0f / grow;   // (each lane's own)
    }
#pragma unroll
    for (int x = 0; x < 2; x++) {
        float16v *c = x == 0 ? dk : dv;
        __syncthreads();
        if (row != 0) {
#pragma unroll
            for (int b = 0; b < W / 32; b++)
#pragma unroll
                for (int i = 0; i < 4; i++) sums[(4 * b + i) * 64] = float4v{c[b][4 * i], c[b][4 * i + 1], c[b][4 * i + 2], c[b][4 * i + 3]};
        }
        __syncthreads();
        if (row == 0 && valid) {
            T *out = (T *)row_of<T>(x == 0 ? l.a.dk : l.a.dv, token, kv);
            float *part = l.parts + ((((int64_t)split * 2 + x) * l.a.kv_heads + kv) * l.tokens + token) * dim;
#pragma unroll
            for (int b = 0; b < W / 32; b++) {
#pragma unroll
                for (int i = 0; i < 16; i++) c[b][i] += sums[(4 * b + i / 4) * 64][i % 4];
                if (l.splits > 1) put_part(part, c[b], b, x == 0 ? l.a.scale * lower : lower, dim);
                else put_rows<T>(out, c[b], b, x == 0 ? l.a.scale * lower : lower, dim);
            }
        }
    }
}

static int launch(const void *kernel, int64_t blocks, const AttendLaunch &l, void *stream, int threads = kThreads)
{
    AttendLaunch copy = l;
    void *args[] = {&copy};
    const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)blocks), dim3(threads), args, 0, (hipStream_t)stream);
    if (e != hipSuccess) (void)hipGetLastError();
    return (int)e;
}

// heads of up to 64 run in tiles 64 wide: half the work of 128
#define ATTEND_KERNEL(name) (l.a.type == TESSEL_BF16 ? (l.a.dim <= 64 ? (const void *)name<bf16, 64> : (const void *)name<bf16, 128>) \
                                                     : (l.a.dim <= 64 ? (const void *)name<f16, 64> : (const void *)name<f16, 128>))

// Splits of a launch's tiles.  The longest tile alone takes `longest` steps of some `step` us, all together `total`, `resident` of them at once; each
// split leaves `bytes`, which are written and read again at some 4.5 GB/ms, and the join is a launch more.  The number with the least
// of the sum, none of fewer than four steps.  (The times of a step and the numbers of resident workgroups are those of heads of 128; narrower ones go by
// them too.  2 heads of 128 over 4096 tokens: forward 107 -> 39 us, and with the backward pass 373 -> 133; 8
// heads over 8192: 220 -> 187 and 801 -> 734; with 32 nothing is split.)
int attend_splits(int64_t longest, int64_t total, int resident, double step, double bytes)
{
    int best = 1;
    double least = 1e30;
    for (int64_t s = 1; s <= std::max<int64_t>(1, longest / 4) && s <= 64; s++) {
        const double us = step * std::max((double)((longest + s - 1) / s), (double)total / resident) + (s > 1 ? 4.0 + s * bytes * 2 / 4.5e6 : 0.0);
        if (us < least) {
            least = us;
            best = (int)s;
        }
    }
    return best;
}

static int join(const AttendLaunch &l, bool forward, const tessel_heads &first, const tessel_heads *second, int heads, int steps_by, void *stream)
{
    AttendLaunch copy = l;
    tessel_heads x = first, y = second ? *second : first;
    bool turned = second != nullptr;
    void *args[] = {&copy, &x, &y, &heads, &steps_by, &turned};
    const void *kernel = l.a.type == TESSEL_BF16 ? (forward ? (const void *)attend_join_kernel<bf16, true> : (const void *)attend_join_kernel<bf16, false>)
                                                 : (forward ? (const void *)attend_join_kernel<f16, true> : (const void *)attend_join_kernel<f16, false>);
    const dim3 grid((unsigned)(l.num_tiles * heads * (kAttendRows / kJoinRows)), second ? 2 : 1);
    const hipError_t e = hipLaunchKernel(kernel, grid, dim3(kThreads), args, 0, (hipStream_t)stream);
    if (e != hipSuccess) (void)hipGetLastError();
    return (int)e;
}

int launch_attend(const AttendLaunch &l, void *stream)
{
    int e = launch(ATTEND_KERNEL(attend_kernel), (int64_t)l.num_tiles * l.a.heads * l.splits, l, stream);
    if (e == 0 && l.splits > 1) e = join(l, true, l.a.o, nullptr, l.a.heads, 1, stream);
    return e;
}

int launch_attend_dq(const AttendLaunch &l, void *stream)
{
    int e = launch(ATTEND_KERNEL(attend_dq_kernel), (int64_t)l.num_tiles * l.a.heads * l.splits, l, stream);
    if (e == 0 && l.splits > 1) e = join(l, false, l.a.dq, nullptr, l.a.heads, 1, stream);
    return e;
}

int launch_attend_dkv(const AttendLaunch &l, void *stream)
{
    int e = launch(ATTEND_KERNEL(attend_dkv_kernel), (int64_t)l.num_tiles * l.a.kv_heads * l.splits, l, stream, kDkvThreads);
    if (e == 0 && l.splits > 1) e = join(l, false, l.a.dk, &l.a.dv, l.a.kv_heads, l.a.heads / l.a.kv_heads, stream);
    return e;
}

}  // namespace tessel
