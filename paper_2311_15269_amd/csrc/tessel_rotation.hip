// The norms of queries and keys for each head with the rotation by position, forward and backward (formulas: include/tessel_block_ops.h).
//
// A head's pairs of channels lie in the registers of a group of lanes, V pairs a lane, from its one read to its one write; a wave takes as many heads of a
// token as it has groups, several tokens where these have few heads, and goes on to the next heads.  The sines and cosines of its tokens
// it works out first, one a lane, and passes them around through LDS: all heads of a token share them.  Backward, a lane adds up the
// gradients of w for its channels over all that its wave goes over; then groups, waves and, by a second kernel, workgroups, in order.
//
// Bound by memory: 8192 tokens of 32 + 8 heads of 128 bf16 forward 33 us (168 MB, 5.1 TB/s; a copy of as much by the dropout's kernel 26, by the library's 29.5, and this kernel's
// own without norms and angles 32: the way it goes through memory, not its arithmetic), backward 54 (252 MB, 4.7 TB/s: 16 waves a compute unit have too little
// under way; registers allow no more, and reads a step ahead cost more registers than they give, 67 us) and 4.6 for the second kernel.  One token
// takes 3.4 us, a launch.
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
    float    share;              // 1 / dim
};

template <typename T, int V> struct Some {
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <typename T> struct Some<T, 1> {
    typedef T type;
};

// sum over the group of lanes; all of them get the same bits.  GROUP: 2^GROUP lanes, or as many as `group` says
template <int CTRL>
__device__ __forceinline__ float plus_lane(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 15, 15, true));
}
template <int GROUP>
__device__ __forceinline__ float group_sum(float v, int group)
{
    if (GROUP >= 0) group = GROUP;
    if (group > 0) v = plus_lane<0xB1>(v);                       // neighbours
    if (group > 1) v = plus_lane<0x4E>(v);                       // pairs of a quad
    if (group > 2) v = plus_lane<0x141>(v);                      // quads of eight lanes, mirrored
    if (group > 3) v = plus_lane<0x140>(v);                      // halves of sixteen
    if (group > 4) v += __shfl_xor(v, 16);
    if (group > 5) v += __shfl_xor(v, 32);
    return v;
}

// 1 / sqrt(v) by the instruction (one step of rounding off), which takes subnormal numbers for nought
__device__ __forceinline__ float over_root(float v)
{
    const bool small = v < 0x1p-96f;
    return __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v) * (small ? 0x1p32f : 1.0f);
}

// An angle in turns, less whole ones, for such as are far: product and quotient are taken in two parts of 64 bits each, what the first rounds off in the second.  Up to 2^70
// radians that is off by less than 2^-30 of a turn, where the product alone is by 2^-53 of the angle, an eighth of a radian at 2^50.  (A product that were contracted
// with what is taken from it would count its rounding twice.)
__device__ __forceinline__ double far_turns(double position, double frequency)
{
#pragma clang fp contract(off)
    constexpr double kOver = 0x1.45f306dc9c883p-3, kMore = -0x1.6b01ec5417056p-57;            // 1 / (2 pi), to 2^-107 of it
    const double angle = position * frequency, rest = fma(position, frequency, -angle), turns = angle * kOver;
    const double more = fma(angle, kOver, -turns) + (angle * kMore + rest * kOver), part = (turns - rint(turns)) + (more - rint(more));
    return part - rint(part);
}

// sines and cosines of a wave's tokens
__device__ __forceinline__ void angles(const tessel_rotation &a, int64_t token, int tokens, float *cosine, float *sine)
{
    const int half = a.turning / 2;
    for (int i = threadIdx.x & 63; i < tokens * half; i += 64) {
        const int t = i / half, p = i - t * half;
        const int64_t n = min(token + t, a.tokens - 1);
        const double position = a.index_type == TESSEL_I64 ? (double)((const int64_t *)a.position)[n] : (double)((const int32_t *)a.position)[n];
        double turns = position * a.frequency[p] * 0.15915494309189535;                  // angle / (2 pi), off by up to 2^-51 of it: 2^-29 where it is near
        const double whole = rint(turns);
        if (__builtin_expect(fabs(turns) < 0x1p22, 1)) {
            turns -= whole;
        } else {                                                 // the position in two parts, which 64 bits hold as they are
            const int64_t far = a.index_type == TESSEL_I64 ? ((const int64_t *)a.position)[n] : ((const int32_t *)a.position)[n];
            turns = far_turns((double)(far >> 32) * 0x1p32, a.frequency[p]) + far_turns((double)(uint32_t)far, a.frequency[p]);
            turns -= rint(turns);
        }
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        cosine[i] = c;
        sine[i] = s;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // (the wave's own LDS: no barrier)
}

// What a lane has of a head: channels first[k] .. + V - 1 and second[k] .. + V - 1 of chunk k, V pairs, first those that turn, then the others.  Pair j are the j-th of both; where
// neighbours are paired (NEAR), of which a chunk's channels are 2 V in a row, two in a row.  Channels that do not turn are paired alike.  A chunk that would pass the last of
// its pairs starts before it, at what other lanes have too (RAGGED): its first `skip` pairs count nothing, and both lanes write the same.
template <int V, int CHUNKS, bool NEAR, bool RAGGED>
struct Mine {
    int  first[CHUNKS], second[CHUNKS], pair[CHUNKS], skip[CHUNKS];
    bool on[CHUNKS], turns[CHUNKS];
    __device__ __forceinline__ Mine(const tessel_rotation &a, int lane, int lanes)
    {
        const int half = a.turning / 2, rest = a.dim / 2 - half, turning = (half + V - 1) / V, chunks = turning + (rest + V - 1) / V;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            const int c = min(lane + k * lanes, chunks - 1);
            on[k] = lane + k * lanes < chunks;
            turns[k] = c < turning;
            const int at = V * (turns[k] ? c : c - turning), pairs = turns[k] ? half : rest, start = RAGGED ? min(at, pairs - V) : at;
            skip[k] = at - start;
            pair[k] = turns[k] ? start : 0;
            first[k] = (turns[k] ? 0 : a.turning) + (NEAR ? 2 * start : start);
            second[k] = first[k] + (NEAR ? V : pairs);
        }
    }
    // does value j of the first V or of the second (h) count
    __device__ __forceinline__ bool counts(int k, int h, int j) const { return !RAGGED || (NEAR ? (h * V + j) / 2 : j) >= skip[k]; }
};

// a chunk as it is in memory, in one piece where it lies in one
template <typename T, int V, bool NEAR>
struct Raw {
    static constexpr int kPieces = NEAR ? 1 : 2, kEach = NEAR ? 2 * V : V;
    typedef typename Some<T, kEach>::type Piece;
    Piece v[kPieces];
    __device__ __forceinline__ void read(const T *first, const T *second)
    {
        v[0] = *(const Piece *)first;
        if constexpr (!NEAR) v[1] = *(const Piece *)second;
    }
    __device__ __forceinline__ void write(T *first, T *second) const
    {
        *(Piece *)first = v[0];
        if constexpr (!NEAR) *(Piece *)second = v[1];
    }
    // in 32 bits, noughts where they do not count
    __device__ __forceinline__ void take(float (&x)[2][V], bool counts) const
    {
#pragma unroll
        for (int e = 0; e < 2 * V; e++) {
            float f;
            if constexpr (kEach == 1) f = (float)v[e];
            else f = (float)v[e / kEach][e % kEach];
            x[e / V][e % V] = counts ? f : 0.0f;
        }
    }
    __device__ __forceinline__ void round(const float (&x)[2][V])
    {
#pragma unroll
        for (int e = 0; e < 2 * V; e++) {
            if constexpr (kEach == 1) v[e] = (T)x[e / V][e % V];
            else v[e / kEach][e % kEach] = (T)x[e / V][e % V];
        }
    }
};
template <int V>
__device__ __forceinline__ void get(float *v, const float *from)
{
#pragma unroll
    for (int j = 0; j < V; j++) v[j] = from[j];
}

// a chunk turned by its angles, or with SIGN -1 back
template <int V, bool NEAR, int SIGN>
__device__ __forceinline__ void turn(float (&x)[2][V], const float *c, const float *s)
{
#pragma unroll
    for (int j = 0; j < V; j++) {
        float &a = NEAR ? x[2 * j / V][2 * j % V] : x[0][j], &b = NEAR ? x[(2 * j + 1) / V][(2 * j + 1) % V] : x[1][j];
        const float p = a, q = b;
        a = SIGN > 0 ? p * c[j] - q * s[j] : p * c[j] + q * s[j];
        b = SIGN > 0 ? p * s[j] + q * c[j] : q * c[j] - p * s[j];
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

// Where a lane's chunks of a tensor's heads are: those of its first head of a token, and the way from one step's to the next.  A lane that has no head in
// the last step has the one before it again, or in the first the last head.
template <typename T, int CHUNKS>
struct Chunks {
    T      *p[CHUNKS][2];
    int64_t by;
    template <typename M>
    __device__ __forceinline__ void set(const tessel_heads &h, int64_t token, int head, const M &mine, int heads)
    {
        T *z = (T *)h.data + token * h.token_stride + head * h.head_stride;
        by = h.head_stride << heads;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            p[k][0] = z + mine.first[k];
            p[k][1] = z + mine.second[k];
        }
    }
    // the way to step s; `full`: every lane has a head there
    __device__ __forceinline__ int64_t way(int s, bool full, bool there) const { return full || there ? s * by : max(s - 1, 0) * by; }
};

// the weights of a lane's channels
template <int V, int CHUNKS, typename M>
__device__ __forceinline__ void weights(float (&w)[CHUNKS][2][V], const float *from, const M &mine)
{
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        get<V>(w[k][0], from + mine.first[k]);
        get<V>(w[k][1], from + mine.second[k]);
    }
}

template <typename T, int V, int CHUNKS, int GROUP, bool NEAR, bool RAGGED>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateLaunch l)
{
    __shared__ __attribute__((aligned(16))) float table[kWaves][2][64 * V * CHUNKS];
    const tessel_rotation &a = l.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tokens = 64 >> l.group >> l.heads;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave;
    if (unit >= l.units) return;
    const Turn at(l, unit, tokens);
    const Mine<V, CHUNKS, NEAR, RAGGED> mine(a, lane & ((1 << l.group) - 1), 1 << l.group);
    const int slot = lane >> l.group, head = slot & ((1 << l.heads) - 1), which = slot >> l.heads;
    const bool there = at.token + which < a.tokens;
    const int64_t token = min(at.token + which, a.tokens - 1);
    angles(a, at.token, tokens, table[wave][0], table[wave][1]);
    float c[CHUNKS][V], s[CHUNKS][V], w[CHUNKS][2][V];
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
        get<V>(c[k], table[wave][0] + which * (a.turning / 2) + mine.pair[k]);
        get<V>(s[k], table[wave][1] + which * (a.turning / 2) + mine.pair[k]);
    }
    Chunks<const T, CHUNKS> z;
    Chunks<T, CHUNKS> o;
    for (int i = at.begin; i < at.end; i++) {
        const bool key = i >= l.steps_q;
        const int step = key ? i - l.steps_q : i, all = key ? a.kv_heads : a.heads;
        const bool full = (step + 1) << l.heads <= all, counts = full || (step << l.heads) + head < all;
        if (i == at.begin || i == l.steps_q) {
            z.set(key ? a.k : a.q, token, min(head, all - 1), mine, l.heads);
            o.set(key ? a.k_out : a.q_out, token, min(head, all - 1), mine, l.heads);
            if (a.wq) weights(w, key ? a.wk : a.wq, mine);
        }
        const int64_t way = z.way(step, full, counts), back = o.way(step, full, counts);
        Raw<T, V, NEAR> raw[CHUNKS];
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) raw[k].read(z.p[k][0] + way, z.p[k][1] + way);
        float x[CHUNKS][2][V], sum = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) raw[k].take(x[k], mine.on[k]);
        if (a.wq) {
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int j = 0; j < V; j++) sum += mine.counts(k, h, j) ? x[k][h][j] * x[k][h][j] : 0.0f;
            const float over = over_root(group_sum<GROUP>(sum, l.group) * l.share + a.eps);
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int j = 0; j < V; j++) x[k][h][j] *= over * w[k][h][j];
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; k++) {
            if (mine.turns[k]) turn<V, NEAR, 1>(x[k], c[k], s[k]);
            if (there && counts && mine.on[k]) {
                raw[k].round(x[k]);
                raw[k].write(o.p[k][0] + back, o.p[k][1] + back);
            }
        }
    }
}

template <typename T, int V, int CHUNKS, int GROUP, bool NEAR, bool RAGGED>
__global__ __launch_bounds__(kThreads) void rotate_backward_kernel(RotateLaunch l)
{
    __shared__ __attribute__((aligned(16))) float table[kWaves][2][64 * V * CHUNKS];
    __shared__ float sums[kWaves][2][256];
    const tessel_rotation &a = l.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tokens = 64 >> l.group >> l.heads;
    const Mine<V, CHUNKS, NEAR, RAGGED> mine(a, lane & ((1 << l.group) - 1), 1 << l.group);
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
            get<V>(c[k], table[wave][0] + which * (a.turning / 2) + mine.pair[k]);
            get<V>(s[k], table[wave][1] + which * (a.turning / 2) + mine.pair[k]);
        }
        Chunks<const T, CHUNKS> z, g;
        Chunks<T, CHUNKS> o;
        for (int i = at.begin; i < at.end; i++) {
            const bool key = i >= l.steps_q;
            const int step = key ? i - l.steps_q : i, all = key ? a.kv_heads : a.heads;
            const bool full = (step + 1) << l.heads <= all, counts = full || (step << l.heads) + head < all;
            if (i == at.begin || i == l.steps_q) {
                z.set(key ? a.k : a.q, token, min(head, all - 1), mine, l.heads);
                g.set(key ? a.dk_out : a.dq_out, token, min(head, all - 1), mine, l.heads);
                o.set(key ? a.dk : a.dq, token, min(head, all - 1), mine, l.heads);
                if (a.wq) weights(w, key ? a.wk : a.wq, mine);
            }
            const int64_t way = z.way(step, full, counts), down = g.way(step, full, counts), back = o.way(step, full, counts);
            Raw<T, V, NEAR> raw[CHUNKS], grad[CHUNKS];
#pragma unroll
            for (int k = 0; k < CHUNKS; k++) {
                raw[k].read(z.p[k][0] + way, z.p[k][1] + way);
                grad[k].read(g.p[k][0] + down, g.p[k][1] + down);
            }
            // (heads and channels that are not there are noughts, which add nothing to the gradients of w)
            float x[CHUNKS][2][V], d[CHUNKS][2][V], sum = 0;
#pragma unroll
            for (int k = 0; k < CHUNKS; k++) {
                raw[k].take(x[k], there && counts && mine.on[k]);
                grad[k].take(d[k], there && counts && mine.on[k]);
                if (mine.turns[k]) turn<V, NEAR, -1>(d[k], c[k], s[k]);
            }
            if (a.wq) {
#pragma unroll
                for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int j = 0; j < V; j++) sum += mine.counts(k, h, j) ? x[k][h][j] * x[k][h][j] : 0.0f;
                float over = over_root(group_sum<GROUP>(sum, l.group) * l.share + a.eps);
                over = there && counts ? over : 0.0f;
                sum = 0;
                const auto add = [&](float (&to)[CHUNKS][2][V]) {
#pragma unroll
                    for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                        for (int h = 0; h < 2; h++)
#pragma unroll
                            for (int j = 0; j < V; j++) {
                                x[k][h][j] *= over;
                                to[k][h][j] += d[k][h][j] * x[k][h][j];
                                d[k][h][j] *= w[k][h][j];
                                sum += mine.counts(k, h, j) ? d[k][h][j] * x[k][h][j] : 0.0f;
                            }
                };
                if (key) add(dw[1]);
                else add(dw[0]);
                const float mean = group_sum<GROUP>(sum, l.group) * l.share;
#pragma unroll
                for (int k = 0; k < CHUNKS; k++)
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int j = 0; j < V; j++) d[k][h][j] = over * (d[k][h][j] - x[k][h][j] * mean);
            }
#pragma unroll
            for (int k = 0; k < CHUNKS; k++)
                if (there && counts && mine.on[k]) {
                    raw[k].round(d[k]);
                    raw[k].write(o.p[k][0] + back, o.p[k][1] + back);
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
                    if (slot == 0 && mine.on[k] && mine.counts(k, h, j)) sums[wave][i][(h ? mine.second[k] : mine.first[k]) + j] = v;
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

// sums of the workgroups' parts: sixteen channels a workgroup, four parts a wave at a time
__global__ __launch_bounds__(1024) void rotate_sum_kernel(RotateLaunch l)
{
    __shared__ float sums[16][16];
    const tessel_rotation &a = l.a;
    const int which = blockIdx.y, lane = threadIdx.x & 63, place = lane & 15, col = blockIdx.x * 16 + place, wave = threadIdx.x >> 6;
    float sum = 0;
    if (col < a.dim)
#pragma unroll 8
        for (int p = wave * 4 + (lane >> 4); p < l.num_parts; p += 64) sum += l.parts[((int64_t)p * 2 + which) * a.dim + col];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16) sums[wave][place] = sum;
    __syncthreads();
    if (threadIdx.x >= 16 || col >= a.dim) return;
    sum = 0;
#pragma unroll
    for (int w = 0; w < 16; w++) sum += sums[w][place];
    float *out = (which == 0 ? a.dwq : a.dwk) + col;
    *out = a.accumulate ? *out + sum : sum;
}

// Pairs a lane: four where those that turn and those that do not are each none or four at least, else one.  (Eight leave too few registers: 8192 tokens of
// 32 + 8 heads of 128 bf16 66 instead of 56 us backward, 33 forward either way.)
static int values_of(const tessel_rotation &a)
{
    const int turns = a.turning / 2, rest = (a.dim - a.turning) / 2;
    return (turns == 0 || turns >= 4) && (rest == 0 || rest >= 4) ? 4 : 1;
}
static int chunks_of(const tessel_rotation &a)
{
    const int v = values_of(a), turns = a.turning / 2, rest = (a.dim - a.turning) / 2;
    return (turns + v - 1) / v + (rest + v - 1) / v;
}

static RotateLaunch rotate_launch(const tessel_rotation &a)
{
    RotateLaunch l = {};
    l.a = a;
    const int chunks = chunks_of(a);
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
    l.share = 1.0f / a.dim;
    return l;
}

int64_t rotate_waves(const tessel_rotation &a) { return rotate_launch(a).units; }
int rotate_parts(const tessel_rotation &a) { return (int)std::min<int64_t>((rotate_launch(a).units + kWaves - 1) / kWaves, 1024); }

template <typename T, bool NEAR>
static const void *rotate_of(const tessel_rotation &a, bool back)
{
#define PICK(V, K, G, R) (back ? (const void *)rotate_backward_kernel<T, V, K, G, NEAR, R> : (const void *)rotate_kernel<T, V, K, G, NEAR, R>)
    if (values_of(a) == 1) return a.dim > 128 ? PICK(1, 2, -1, false) : PICK(1, 1, -1, false);
    if (a.turning % 8 || (a.dim - a.turning) % 8) return PICK(4, 1, -1, true);
    // (heads of 72 to 128 and of 40 to 64 channels without a branch for each step of their sums)
    return a.dim > 128 || a.dim <= 32 ? PICK(4, 1, -1, false) : a.dim > 64 ? PICK(4, 1, 4, false) : PICK(4, 1, 3, false);
#undef PICK
}
template <typename T>
static const void *rotate_of(const tessel_rotation &a, bool back)
{
    return a.neighbours || a.turning == 0 ? rotate_of<T, true>(a, back) : rotate_of<T, false>(a, back);      // (where none turns, in one piece)
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
        e = launched(hipLaunchKernel((const void *)rotate_sum_kernel, dim3((unsigned)((a.dim + 15) / 16), 2), dim3(1024), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
