// The embedding of a shard of the vocabulary, forward and backward (formulas: include/tessel_block_ops.h).
//
// Forward: eight channels of a token a lane.  Backward: a workgroup for every row of the table looks through all tokens for its own, in order.
#include "tessel_draw.h"

namespace tessel {

constexpr int kThreads = 256;

// the row of the table that token t takes, -1 if there is none
__device__ __forceinline__ int row_at(const tessel_embedding &a, int64_t t)
{
    const int64_t v = a.index_type == TESSEL_I64 ? ((const int64_t *)a.token)[t] : ((const int32_t *)a.token)[t];
    return v >= a.first && v - a.first < a.rows ? (int)(v - a.first) : -1;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void embed_kernel(tessel_embedding a, DropLaunch d)
{
    const uint32_t per = (uint32_t)(((int64_t)a.channels + 7) / 8);
    const uint64_t n = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = (int64_t)(n / per);
    const int col = (int)(n % per) * 8;
    if (t >= a.tokens) return;
    const int row = row_at(a, t);
    float v[8] = {};
    if (row >= 0) {
        load8<T>(v, (const T *)a.table.data + row * a.table.stride, col, a.channels);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] *= a.scale;
        if (d.least) drop8(v, d, number_of(d), (uint32_t)t, col);
    }
    store8<T>((T *)a.out.data + t * a.out.stride, v, col, a.channels);
}

// Backward: the places of a batch sorted by row, those of a row in ascending order (sort_kernel); sums over runs of so many sorted places
// (sum_kernel); sums of what the runs left of rows that go on from one run into the next, and rows that no token asked for (join_kernel).
struct EmbedLaunch {
    tessel_embedding a;
    DropLaunch d;
    int32_t *place, *row;        // [tokens] sorted: place in the batch, row of the table
    int32_t *total;              // how many of them
    int32_t *count;              // [buckets][bins]: tokens of row bin * buckets + bucket
    float   *parts;              // [runs][2][channels]: of the row that a run begins within, and of the one that goes on behind it
    int32_t  bins, shift;        // buckets = 2^shift
    int32_t  run, runs;          // sorted places a run
    int32_t  lanes;              // that hold a run's columns: a power of two up to 256, eight columns each
};

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kEach = 4, kTile = kSortThreads * kEach;
constexpr int kMostBins = 4096;

// rows of the table for tokens t .. t + 3, -1 where there is none
template <typename I>
__device__ __forceinline__ void rows4(const tessel_embedding &a, int64_t t, int (&v)[kEach])
{
    typedef I V __attribute__((ext_vector_type(4), aligned(sizeof(I))));
    const I *p = (const I *)a.token;
    V w;
    if (t + kEach <= a.tokens) {
        w = *(const V *)(p + t);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; j++) w[j] = t + j < a.tokens ? p[t + j] : (I)-1;
    }
#pragma unroll
    for (int j = 0; j < kEach; j++) {
        const int64_t n = w[j];
        v[j] = n >= a.first && n - a.first < a.rows ? (int)(n - a.first) : -1;
    }
}

__device__ __forceinline__ int below(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u)); }

// A workgroup for each bucket of rows with the same low bits (frequent tokens are neighbours in a vocabulary).  It counts the places of its rows
// and of the buckets before it, and then goes through the batch once more, a tile at a time, and puts its places where they belong.
template <typename I>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(EmbedLaunch l)
{
    __shared__ int cursor[kMostBins];                            // counts, then the place where the next one of a row goes
    __shared__ int list_row[kTile], list_place[kTile];           // this bucket's share of a tile, in order
    __shared__ int sums[2][kSortWaves];
    const tessel_embedding &a = l.a;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6, bucket = blockIdx.x, mask = (1 << l.shift) - 1;
    for (int b = thread; b < l.bins; b += kSortThreads) cursor[b] = 0;
    __syncthreads();
    int before = 0, own = 0;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kTile) {
        int v[kEach];
        rows4<I>(a, t0 + kEach * thread, v);
#pragma unroll
        for (int j = 0; j < kEach; j++) {
            before += v[j] >= 0 && (v[j] & mask) < bucket ? 1 : 0;
            if (v[j] >= 0 && (v[j] & mask) == bucket) {
                own++;
                atomicAdd(&cursor[v[j] >> l.shift], 1);          // (whole numbers: the order does not matter)
            }
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        before += __shfl_xor(before, d);
        own += __shfl_xor(own, d);
    }
    if (lane == 0) {
        sums[0][wave] = before;
        sums[1][wave] = own;
    }
    __syncthreads();
    before = own = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) {
        before += sums[0][w];
        own += sums[1][w];
    }
    if (bucket == mask && thread == 0) *l.total = before + own;
    if (!a.accumulate)
        for (int b = thread; b < l.bins; b += kSortThreads) l.count[(int64_t)bucket * l.bins + b] = cursor[b];
    if (own == 0) return;
    // where each row's places begin: four bins a thread
    __syncthreads();
    int c[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        c[j] = 4 * thread + j < l.bins ? cursor[4 * thread + j] : 0;
        sum += c[j];
    }
    int up = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(up, d);
        if (lane >= d) up += x;
    }
    if (lane == 63) sums[0][wave] = up;
    __syncthreads();
    int at = before + up - sum;
    for (int w = 0; w < wave; w++) at += sums[0][w];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if (4 * thread + j < l.bins) cursor[4 * thread + j] = at;
        at += c[j];
    }
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kTile) {
        int v[kEach], n = 0;
        rows4<I>(a, t0 + kEach * thread, v);
#pragma unroll
        for (int j = 0; j < kEach; j++) {
            if (v[j] >= 0 && (v[j] & mask) != bucket) v[j] = -1;
            n += v[j] >= 0 ? 1 : 0;
        }
        // places before this thread's: n is 0 to 4
        const uint64_t one = __ballot(n & 1), two = __ballot(n & 2), four = __ballot(n & 4);
        int to = below(one) + 2 * below(two) + 4 * below(four);
        __syncthreads();                                         // (the list and the sums of the tile before are done with)
        if (lane == 0) sums[0][wave] = __popcll(one) + 2 * __popcll(two) + 4 * __popcll(four);
        __syncthreads();
        int found = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; w++) {
            to += w < wave ? sums[0][w] : 0;
            found += sums[0][w];
        }
#pragma unroll
        for (int j = 0; j < kEach; j++)
            if (v[j] >= 0) {
                list_row[to] = v[j];
                list_place[to] = (int)(t0 + kEach * thread + j);
                to++;
            }
        __syncthreads();
        for (int first = 0; first < found; first += kSortThreads) {
            // a wave's 64 places: how many of the same row come before, and which lane is the first of the row
            const int i = first + thread, row = i < found ? list_row[i] : -1, bin = row >> l.shift;
            uint64_t same = __ballot(row >= 0);
            for (int b = 0; 1 << b < l.bins; b++) {
                const uint64_t bit = __ballot(bin >> b & 1);
                same &= bin >> b & 1 ? bit : ~bit;
            }
            const int rank = below(same), leader = __ffsll((unsigned long long)same) - 1;
            const int waves = min(kSortWaves, (found - first + 63) / 64);
            int start = 0;
            for (int w = 0; w < waves; w++) {                    // (the waves one after the other: places of a row stay in order)
                if (wave == w && row >= 0 && rank == 0) {
                    start = cursor[bin];
                    cursor[bin] = start + __popcll(same);
                }
                __syncthreads();
            }
            start = __shfl(start, leader < 0 ? 0 : leader);
            if (row >= 0) {
                l.place[start + rank] = list_place[i];
                l.row[start + rank] = row;
            }
        }
    }
}

// what a run left of a row, or all of it
template <bool NARROW>
__device__ __forceinline__ void put_sum(const EmbedLaunch &l, float *to, bool whole, const float *sum, int col)
{
    const tessel_embedding &a = l.a;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = whole ? a.scale * sum[j] : sum[j];
    if (whole && a.accumulate) {
        float old[8];
        load8<float>(old, to, col, a.channels);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] += old[j];
    }
    store8<float>(to, v, col, a.channels);
}

template <typename T, bool NARROW>
__global__ __launch_bounds__(kThreads) void sum_kernel(EmbedLaunch l)
{
    constexpr int kAhead = 8;
    const tessel_embedding &a = l.a;
    int run = blockIdx.x * (kThreads / l.lanes) + threadIdx.x / l.lanes;
    if (l.lanes >= 64) run = __builtin_amdgcn_readfirstlane(run);
    const int col = 8 * (blockIdx.y * l.lanes + threadIdx.x % l.lanes), total = *l.total;
    const int64_t first = (int64_t)run * l.run;
    if (run >= l.runs || first >= total || col >= a.channels) return;
    const uint32_t begin = (uint32_t)first, end = (uint32_t)min(first + l.run, (int64_t)total);
    const uint64_t number = number_of(l.d);
    int row = l.row[begin];
    bool starts = begin == 0 || l.row[begin - 1] != row;         // (the row's first place is in this run)
    float sum[8] = {};
    const auto flush = [&](bool ends) {
        const bool whole = starts && ends;
        put_sum<NARROW>(l, whole ? a.dtable + row * a.dtable_stride : l.parts + ((int64_t)run * 2 + (starts ? 1 : 0)) * a.channels, whole, sum, col);
    };
    for (uint32_t i = begin; i < end; i += kAhead) {
        int r[kAhead], t[kAhead];
        typename Eight<T>::type x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            r[j] = l.row[min(i + j, end - 1)];
            t[j] = l.place[min(i + j, end - 1)];
        }
#pragma unroll
        for (int j = 0; j < kAhead; j++) x[j] = take8<T, NARROW>((const T *)a.d_out.data + t[j] * a.d_out.stride, col, a.channels);
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            if (i + j >= end) break;
            if (r[j] != row) {
                flush(true);
                row = r[j];
                starts = true;
#pragma unroll
                for (int k = 0; k < 8; k++) sum[k] = 0;
            }
            float v[8];
            settle8<T, NARROW>(col, a.channels, x[j]);
            widen8<T>(v, x[j]);
            if (l.d.least) drop8(v, l.d, number, (uint32_t)t[j], col);
#pragma unroll
            for (int k = 0; k < 8; k++) sum[k] += v[k];
        }
    }
    flush(end == (uint32_t)total || l.row[end] != row);
}

// The first workgroups, one for each run and 4 lanes columns: where a row goes on behind the run that it starts in, the sum of what the runs left of it.
// The others, rows that no token asked for.
__global__ __launch_bounds__(kSortThreads) void join_kernel(EmbedLaunch l, int joins, int tiles)
{
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
    __shared__ float4v sums[kSortThreads];
    const tessel_embedding &a = l.a;
    if ((int)blockIdx.x >= joins) {                              // a wave for each row
        const int step = (gridDim.x - joins) * kSortWaves, lane = threadIdx.x & 63;
        for (int64_t row = (int64_t)(blockIdx.x - joins) * kSortWaves + (threadIdx.x >> 6); row < a.rows; row += step) {
            if (l.count[(row & ((1 << l.shift) - 1)) * l.bins + (row >> l.shift)]) continue;
            float *to = a.dtable + row * a.dtable_stride;
            const float zero[8] = {};
            for (int col = 8 * lane; col < a.channels; col += 512) store8<float>(to, zero, col, a.channels);
        }
        return;
    }
    const int run = blockIdx.x / tiles, total = *l.total;
    const int64_t last = ((int64_t)run + 1) * l.run;
    if (last >= total) return;
    const int row = l.row[last - 1], lane = threadIdx.x & 63;
    if (l.row[last] != row) return;
    if (l.row[last - l.run] == row && run > 0 && l.row[last - l.run - 1] == row) return;       // (it does not start here)
    int more = 0;                                                // runs that it goes on in
    for (;;) {
        const int64_t i = (int64_t)(run + 1 + more + lane) * l.run;
        const uint64_t there = __ballot(i < total && l.row[min(i, (int64_t)total - 1)] == row);
        const int n = there == ~0ull ? 64 : __ffsll((unsigned long long)~there) - 1;
        more += n;
        if (n < 64) break;
    }
    const int lanes = 2 * l.lanes, groups = kSortThreads / lanes, group = threadIdx.x / lanes, at = threadIdx.x % lanes;
    const int col = 4 * (blockIdx.x % tiles * lanes + at);
    V sum = {};
    if (col < a.channels) {
        const int whole = min(4, a.channels - col);
        const auto part = [&](int p) {                           // the first of them is the run's own
            const float *from = l.parts + ((int64_t)(run + p) * 2 + (p == 0 ? 1 : 0)) * a.channels + col;
            V v = {};
            if (whole == 4) v = *(const V *)from;
            else
                for (int j = 0; j < whole; j++) v[j] = from[j];
            return v;
        };
#pragma unroll 8
        for (int p = group; p <= more; p += groups) sum += part(p);
    }
    sums[threadIdx.x] = float4v{sum[0], sum[1], sum[2], sum[3]};
    __syncthreads();
    if (group > 0 || col >= a.channels) return;
    for (int g = 1; g < min(groups, more + 1); g++) {
        const float4v v = sums[g * lanes + at];
        sum += V{v[0], v[1], v[2], v[3]};
    }
    float *to = a.dtable + row * a.dtable_stride + col;
    for (int j = 0; j < min(4, a.channels - col); j++) to[j] = (a.accumulate ? to[j] : 0.0f) + a.scale * sum[j];
}

int launch_embed(const tessel_embedding &a, const DropLaunch &d, void *stream)
{
    tessel_embedding aa = a;
    DropLaunch dd = d;
    void *args[] = {&aa, &dd};
    const int64_t lanes = a.tokens * (((int64_t)a.channels + 7) / 8);
#define KERNEL(T) ((const void *)embed_kernel<T>)
    return launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)((lanes + kThreads - 1) / kThreads)), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

static EmbedLaunch embed_launch(const tessel_embedding &a)
{
    EmbedLaunch l = {};
    l.a = a;
    l.shift = 8;
    while (((int64_t)a.rows + (1 << l.shift) - 1) >> l.shift > kMostBins) l.shift++;
    l.bins = (int)(((int64_t)a.rows + (1 << l.shift) - 1) >> l.shift);
    l.lanes = 8;
    while (l.lanes < 256 && 8 * l.lanes < a.channels) l.lanes *= 2;
    // places a run: few enough that the runs fill the GPU, and that there are at most 2048 of them
    const int64_t threads = a.tokens * (((int64_t)a.channels + 7) / 8);
    l.run = 8;
    while (l.run < threads >> 18 || (int64_t)l.run * 2048 < a.tokens) l.run *= 2;
    l.runs = (int)((a.tokens + l.run - 1) / l.run);
    return l;
}

static size_t whole_chunks(int64_t words) { return (size_t)(words + 3) / 4 * 4; }
static size_t counts_of(const tessel_embedding &a, const EmbedLaunch &l) { return a.accumulate ? 0 : whole_chunks((int64_t)l.bins << l.shift); }

size_t embed_workspace(const tessel_embedding &a)
{
    const EmbedLaunch l = embed_launch(a);
    return 4 * (2 * whole_chunks(a.tokens) + 4 + counts_of(a, l) + whole_chunks((int64_t)l.runs * 2 * a.channels));
}

int launch_embed_backward(const tessel_embedding &a, const DropLaunch &d, void *workspace, void *stream)
{
    EmbedLaunch l = embed_launch(a);
    l.d = d;
    l.place = (int32_t *)workspace;
    l.row = l.place + whole_chunks(a.tokens);
    l.total = l.row + whole_chunks(a.tokens);
    l.count = l.total + 4;
    l.parts = (float *)(l.count + counts_of(a, l));
    void *args[] = {&l};
    const void *sort = a.index_type == TESSEL_I64 ? (const void *)sort_kernel<int64_t> : (const void *)sort_kernel<int32_t>;
    int e = launched(hipLaunchKernel(sort, dim3(1u << l.shift), dim3(kSortThreads), args, 0, (hipStream_t)stream));
    if (e == 0 && l.runs > 0) {
        const int each = kThreads / l.lanes;
#define KERNEL(T) (a.channels < 8 ? (const void *)sum_kernel<T, true> : (const void *)sum_kernel<T, false>)
        const dim3 grid((unsigned)((l.runs + each - 1) / each), (unsigned)(((int64_t)a.channels + 8 * l.lanes - 1) / (8 * l.lanes)));
        e = launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), grid, dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
    }
    int tiles = (int)(((int64_t)a.channels + 8 * l.lanes - 1) / (8 * l.lanes)), joins = l.runs > 1 ? l.runs * tiles : 0;
    const int fills = a.accumulate ? 0 : (int)(a.rows / kSortWaves + 1 < 4096 ? a.rows / kSortWaves + 1 : 4096);
    void *more[] = {&l, &joins, &tiles};
    if (e == 0 && joins + fills > 0)
        e = launched(hipLaunchKernel((const void *)join_kernel, dim3((unsigned)(joins + fills)), dim3(kSortThreads), more, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
