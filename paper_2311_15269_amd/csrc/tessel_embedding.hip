// The embedding of a shard of the vocabulary, forward and backward (formulas: include/tessel_block_ops.h).
//
// Forward: a gather, eight channels of a token a lane, scaled and dropped on its way.  Backward: a sum over the tokens of each row.  Adding them up with atomics would
// make their order, and with it the bits, chance; so the places of the batch are sorted by row first, stably, and every sum goes over its places in ascending
// order, in pieces whose bounds, and the order in which they are joined, do not depend on what runs when (but on where the row lies among the shard's others).  The
// sort is by buckets of rows with the same low bits, a workgroup each, which all read the whole batch (T tokens 256 times, from the caches) and need nothing from
// each other: one launch, where a sort by digits takes three a digit.
//
// Bound by memory but for the way through the launches.  Forward, 8192 tokens of 4096 bf16: 17 us (100 MB, 5.8 TB/s), with dropout 21; 16384 of 1024 f16 10.  Backward,
// the same 8192 tokens into 50000 rows of which some 3700 occur: sort 8.8 us, sums and zeros 165 (886 MB, 5.4 TB/s; zeros alone 5.8), join 8; 16384 tokens added
// to 62500 rows of 1024: 10, 18 and 7 us.  512 tokens and fewer in one launch, 2.5 to 13 us.
#include <algorithm>

#include "tessel_draw.h"

namespace tessel {

constexpr int kThreads = 256;

// the row of the table that a token takes, -1 if there is none (one comparison: what is below `first` wraps around)
__device__ __forceinline__ int row_of(const tessel_embedding &a, int64_t token)
{
    const uint64_t row = (uint64_t)token - (uint64_t)a.first;
    return row < (uint64_t)a.rows ? (int)row : -1;
}
__device__ __forceinline__ int row_at(const tessel_embedding &a, int64_t t)
{
    return row_of(a, a.index_type == TESSEL_I64 ? ((const int64_t *)a.token)[t] : ((const int32_t *)a.token)[t]);
}

template <typename T, bool WIDE, int ROWS>
__global__ __launch_bounds__(kThreads) void embed_kernel(tessel_embedding a, DropLaunch d, int lanes)
{
    const Span<WIDE, ROWS> at(a.channels, lanes);
    int row[ROWS];
    typename Eight<T>::type x[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; r++) row[r] = row_at(a, min(at.token + r * at.step, a.tokens - 1));
#pragma unroll
    for (int r = 0; r < ROWS; r++) x[r] = read8<T, !WIDE>((const T *)a.table.data + max(row[r], 0) * a.table.stride, at.col, a.channels);
    const Draw draw(d, a.channels, at.col);
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        const int64_t token = at.token + r * at.step;
        if (token >= a.tokens) break;
        float v[8];
        place8<T, !WIDE>(at.col, a.channels, x[r]);
        widen8<T>(v, x[r]);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = row[r] >= 0 ? v[j] * a.scale : 0.0f;
        if (d.least) draw.apply(v, (uint32_t)token);
        store8<T>((T *)a.out.data + token * a.out.stride, v, at.col, a.channels);
    }
}

// Backward: the places of a batch sorted by row, those of a row in ascending order (sort_kernel); sums over runs of so many sorted places, and zeros in the rows that no
// token asked for (sum_kernel); sums of what the runs left of rows that go on from one run into the next (join_kernel).
struct EmbedLaunch {
    tessel_embedding a;
    DropLaunch d;
    int32_t *place, *row;        // [tokens + 8] sorted: place in the batch, row of the table
    int32_t *total;              // how many of them
    int32_t *count;              // [buckets][bins], where the gradient is written: tokens of row bin * buckets + bucket
    float   *parts;              // [runs][2][part]: of the row that a run begins within, and of the one that goes on behind it
    int64_t  part;               // channels up to the next multiple of eight
    int32_t  bins, shift;        // buckets = 2^shift
    int32_t  run, runs;          // sorted places a run
    int32_t  lanes, tiles;       // that hold a run's columns: a power of two up to 256, eight columns each; of them, to the end of a row
    uint32_t sum_groups;         // workgroups that add up
    uint32_t fill_rows, fill_pieces, fill_lanes;      // zeros: rows a piece, pieces a row (one of the two is one); lanes a row takes
    int64_t  fills;              // pieces in all
};

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSubs = 4, kSub = 4 * kSortThreads, kTile = kSubs * kSub;          // a thread takes four places of each part of a tile
constexpr int kMostBins = 2 * kSortThreads;        // (two workgroups have room on a compute unit)
constexpr int kOften = 256;      // places of a row that is put in place by counting (32768 tokens, nearly all of them one: sort 54 us, without this 74)

__device__ __forceinline__ int below(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u)); }

// sums over the lanes up to and with this one, and their largest value so far (whole numbers from 0 on)
template <typename F>
__device__ __forceinline__ int up_to(int x, F &&f)
{
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 15, 15, false));         // of sixteen lanes: one, two, four and eight back
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 15, 15, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 15, 15, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 15, 15, false));
    x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 10, 15, false));         // the last lane of the sixteen before, to the second and fourth
    return f(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 12, 15, false));      // of the first half, to the second
}
__device__ __forceinline__ int sums_up_to(int x) { return up_to(x, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int most_up_to(int x) { return up_to(x, [](int a, int b) { return max(a, b); }); }

// A thread's places of the tile at t0, sixteen bits: those whose row is in the bucket.  `before`: how many are in the buckets before it, added up.  (No read stands in a
// branch, behind which the compiler would wait for it: behind the last place the last four are read again.  Of four tokens there are more: few_kernel takes batches of up to 256.)
template <typename I>
__device__ __forceinline__ uint32_t tile_places(const EmbedLaunch &l, int64_t t0, uint32_t bucket, int &before)
{
    typedef I V __attribute__((ext_vector_type(4), aligned(sizeof(I))));
    const tessel_embedding &a = l.a;
    const uint32_t buckets = 1u << l.shift;
    V w[kSubs];
#pragma unroll
    for (int s = 0; s < kSubs; s++) {
        const int64_t t = t0 + s * kSub + 4 * (int)threadIdx.x;
        w[s] = *(const V *)((const I *)a.token + min(t, a.tokens - 4));
    }
    uint32_t mine = 0;
#pragma unroll
    for (int s = 0; s < kSubs; s++) {
        const int64_t t = t0 + s * kSub + 4 * (int)threadIdx.x;
        if (t0 + s * kSub >= a.tokens) break;
        uint32_t here = 0;
        int less = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint64_t row = (uint64_t)(int64_t)w[s][j] - (uint64_t)a.first;
            const uint32_t b = row < (uint64_t)a.rows ? (uint32_t)row & (buckets - 1) : buckets;
            here |= b == bucket ? 1u << j : 0u;
            less |= b < bucket ? 1 << j : 0;
        }
        if (__any(t + 4 > a.tokens)) {                           // the last places: of those read again, what is not there
            const int by = (int)min(t - min(t, a.tokens - 4), (int64_t)4), left = (int)min(max(a.tokens - t, (int64_t)0), (int64_t)4);
            here = here >> by & ((1u << left) - 1);
            less = less >> by & ((1 << left) - 1);
        }
        before += __popc(less);
        mine |= here << (4 * s);
    }
    return mine;
}

// A workgroup for each bucket of rows with the same low bits (frequent tokens are neighbours in a vocabulary).  It goes through the batch a tile at a time and lists its
// places in order.  Once to count them by row, and those of the buckets before it; once more to put them where they belong, if not all of them fit the list.
template <typename I>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(EmbedLaunch l)
{
    __shared__ int cursor[kMostBins];                            // counts, then the place where the next one of a row goes
    __shared__ uint16_t list[2][kTile];                          // places behind `base`
    __shared__ int sums[2][kSortWaves], shares[kSubs * kSortWaves];
    static_assert(kSubs * kSortWaves == 64 && kTile <= 1 << 16 && kMostBins <= 1 << 11, "a lane for each wave's share of a part; 16 bits of a place, 11 of a bin");
    const tessel_embedding &a = l.a;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6, bucket = blockIdx.x;
    const bool near = a.tokens <= 1 << 16;                       // (16 bits hold any place)
    const auto row_in = [&](int64_t base, int place) { return row_of(a, ((const I *)a.token)[base + place]); };
    // The tile's places of this bucket to list[0] behind its first `listed`, or in place of these if they would not fit; how many there are.  Through barriers:
    // all are done with an earlier list before it is written, and it is there when this returns.
    const auto find = [&](int64_t t0, int64_t base, int &listed, int &before) {
        uint32_t mine = tile_places<I>(l, t0, (uint32_t)bucket, before);
        int to[kSubs];
#pragma unroll
        for (int s = 0; s < kSubs; s++) {                        // none to four of each thread
            const int n = __popc(mine >> 4 * s & 15u);
            const uint64_t one = __ballot(n & 1), two = __ballot(n & 2), four = __ballot(n & 4);
            to[s] = below(one) + 2 * below(two) + 4 * below(four);
            if (lane == 0) shares[s * kSortWaves + wave] = __popcll(one) + 2 * __popcll(two) + 4 * __popcll(four);
        }
        __syncthreads();
        const int share = shares[lane], through = sums_up_to(share), found = __shfl(through, 63);
        listed = listed + found <= kTile ? listed : 0;
#pragma unroll
        for (int s = 0; s < kSubs; s++) {
            int i = listed + to[s] + __shfl(through - share, s * kSortWaves + wave);
            for (uint32_t m = mine >> 4 * s & 15u; m; m &= m - 1) list[0][i++] = (uint16_t)(t0 - base + s * kSub + 4 * thread + __builtin_ctz(m));
        }
        __syncthreads();
        return found;
    };
    for (int b = thread; b < l.bins; b += kSortThreads) cursor[b] = 0;
    int before = 0, own = 0, listed = 0;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kTile) {
        const int64_t base = near ? 0 : t0;
        if (!near) listed = 0;
        const int found = find(t0, base, listed, before);
        for (int first = 0; first < found; first += kSortThreads) {
            // (whole numbers: the order does not matter.  The first lane's row at once: those of a frequent one would wait for each other at its count)
            const int i = first + thread, row = i < found ? row_in(base, list[0][listed + i]) : -1, one = __builtin_amdgcn_readfirstlane(row);
            const int n = __popcll(__ballot(row == one));
            if (row >= 0 && (row != one || lane == 0)) atomicAdd(&cursor[row >> l.shift], row == one ? n : 1);
        }
        own += found;
        listed += found;
    }
    const bool all = near && listed == own;                      // the list holds every place
    before = sums_up_to(before);
    if (lane == 63) sums[0][wave] = before;
    __syncthreads();
    before = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) before += sums[0][w];
    if (bucket == (1 << l.shift) - 1 && thread == 0) *l.total = before + own;
    if (!a.accumulate)
        for (int b = thread; b < l.bins; b += kSortThreads) l.count[(int64_t)bucket * l.bins + b] = cursor[b];
    if (own == 0) return;
    // where each row's places begin: two bins a thread; and the most frequent row
    int c[2], sum = 0, top = 0;
#pragma unroll
    for (int j = 0; j < 2; j++) {
        c[j] = 2 * thread + j < l.bins ? cursor[2 * thread + j] : 0;
        sum += c[j];
        top = max(top, min(c[j], (1 << 20) - 1) << 11 | (2 * thread + j));
    }
    const int up = sums_up_to(sum);
    top = most_up_to(top);
    __syncthreads();                                             // (all are done with the counts and sums)
    if (lane == 63) {
        sums[0][wave] = up;
        sums[1][wave] = top;
    }
    __syncthreads();
    int at = before + up - sum;
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) {
        at += w < wave ? sums[0][w] : 0;
        top = max(top, sums[1][w]);
    }
#pragma unroll
    for (int j = 0; j < 2; j++) {
        if (2 * thread + j < l.bins) cursor[2 * thread + j] = at;
        at += c[j];
    }
    __syncthreads();
    // A row of many places: they are put in place by counting alone, and only the others go through the steps below, wave by wave.
    const int often = top >> 11 >= kOften ? (top & 2047) << l.shift | bucket : -2;
    int often_at = often >= 0 ? cursor[often >> l.shift] : 0;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kTile) {
        const int64_t base = all ? 0 : t0;
        int found = own, none = 0, from = 0;
        if (!all) found = find(t0, base, from, none);
        int which = 0;
        if (often >= 0) {
            int others = 0;
            for (int first = 0; first < found; first += kSortThreads) {
                const int i = first + thread, place = i < found ? list[0][i] : 0, row = i < found ? row_in(base, place) : -1;
                const uint64_t same = __ballot(row == often), rest = __ballot(row >= 0 && row != often);
                if (lane == 0) {
                    sums[0][wave] = __popcll(same);
                    sums[1][wave] = __popcll(rest);
                }
                __syncthreads();
                int to = often_at + below(same), rest_to = others + below(rest);
#pragma unroll
                for (int w = 0; w < kSortWaves; w++) {
                    to += w < wave ? sums[0][w] : 0;
                    rest_to += w < wave ? sums[1][w] : 0;
                    often_at += sums[0][w];
                    others += sums[1][w];
                }
                if (row == often) {
                    l.place[to] = (int)(base + place);
                    l.row[to] = often;
                } else if (row >= 0) {
                    list[1][rest_to] = (uint16_t)place;
                }
                __syncthreads();
            }
            which = 1;
            found = others;
        }
        for (int first = 0; first < found; first += kSortThreads) {
            // a wave's 64 places: how many of the same row come before, and which lane is the first of the row
            const int i = first + thread;
            const bool there = i < found;
            const int place = there ? list[which][i] : 0, row = there ? row_in(base, place) : bucket, bin = row >> l.shift;
            uint64_t same = __ballot(there);
            for (int b = 0; 1 << b < l.bins; b++) {
                const uint64_t bit = __ballot(bin >> b & 1);
                same &= bin >> b & 1 ? bit : ~bit;
            }
            const int rank = below(same), leader = max(0, __ffsll((unsigned long long)same) - 1);
            const int waves = min(kSortWaves, (found - first + 63) / 64);
            int start = 0;
            for (int w = 0; w < waves; w++) {                    // (the waves one after the other: places of a row stay in order)
                if (wave == w && there && rank == 0) {
                    start = cursor[bin];
                    cursor[bin] = start + __popcll(same);
                }
                __syncthreads();
            }
            start = __shfl(start, leader);
            if (there) {
                l.place[start + rank] = (int)(base + place);
                l.row[start + rank] = row;
            }
        }
        if (all) break;
    }
}

constexpr int kFill = 4096;      // values that a workgroup fills with zeros at most (100000 rows of 264 channels 18 us, 200000 of 40 10.6; four times as many a workgroup 19 and 14)

// Zeros in the rows of a piece that no token asked for; neighbouring workgroups write neighbouring pieces.
struct Piece {
    int64_t row;                 // the first of fill_rows
    int     begin, end;          // columns
    __device__ __forceinline__ Piece(const EmbedLaunch &l, int64_t piece) : row(piece / l.fill_pieces * l.fill_rows), begin((int)(piece % l.fill_pieces) * kFill)
    {
        end = (int)min((int64_t)l.a.channels, (int64_t)begin + kFill);
    }
};
template <int THREADS, typename F>
__device__ __forceinline__ void fill(const EmbedLaunch &l, const Piece &p, F &&asked)
{
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
    const tessel_embedding &a = l.a;
    const int lanes = l.fill_lanes, lane = threadIdx.x % lanes;
    for (int r = threadIdx.x / lanes; r < (int)l.fill_rows; r += THREADS / lanes) {
        if (p.row + r >= a.rows || asked(r)) continue;
        float *to = a.dtable + (p.row + r) * a.dtable_stride;
        int col = p.begin + 4 * lane;
        for (; col + 4 <= p.end; col += 4 * lanes) *(V *)(to + col) = V{};
        for (int j = col; j < p.end; j++) to[j] = 0.0f;
    }
}

// a row's whole sum
__device__ __forceinline__ void put_row(const tessel_embedding &a, int row, float (&sum)[8], int col)
{
    float *to = a.dtable + row * a.dtable_stride, old[8] = {};
    if (a.accumulate) load8<float>(old, to, col, a.channels);
#pragma unroll
    for (int j = 0; j < 8; j++) sum[j] = old[j] + a.scale * sum[j];
    store8<float>(to, sum, col, a.channels);
}

// A batch of few tokens in one launch.  A workgroup for each token and 512 columns: its waves look which tokens have the same row, 64 each; that of the first of these adds
// them up, a wave its share of the tokens, and the waves' sums in order.  Behind them workgroups that fill the other rows.  WAVES: as many as the tokens take
template <typename T, int WAVES, bool NARROW>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(EmbedLaunch l)
{
    __shared__ uint64_t found[WAVES];
    __shared__ uint32_t seen[kFill / 32];
    __shared__ float4v sums[WAVES][2][64];
    const tessel_embedding &a = l.a;
    const int thread = threadIdx.x, lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int mine = thread < a.tokens ? row_at(a, thread) : -1;
    if (blockIdx.x >= l.sum_groups) {
        for (int64_t piece = blockIdx.x - l.sum_groups; piece < l.fills; piece += gridDim.x - l.sum_groups) {
            const Piece p(l, piece);
            for (int n = thread; n < kFill / 32; n += 64 * WAVES) seen[n] = 0;
            __syncthreads();
            if (mine >= p.row && mine < p.row + l.fill_rows) atomicOr(&seen[(mine - p.row) / 32], 1u << (mine - p.row) % 32);
            __syncthreads();
            fill<64 * WAVES>(l, p, [&](int r) { return seen[r / 32] >> r % 32 & 1; });
            __syncthreads();
        }
        return;
    }
    const int token = blockIdx.x / l.tiles, col = 8 * (blockIdx.x % l.tiles * 64 + lane), row = row_at(a, token);
    if (row < 0) return;
    uint64_t same = __ballot(mine == row);
    if (lane == 0) found[wave] = same;
    __syncthreads();
    int first = 0;
    while (found[first] == 0) first++;                           // (one of them is this token)
    if (64 * first + __builtin_ctzll(found[first]) != token) return;
    const Draw draw(l.d, a.channels, col);
    float sum[8] = {};
    while (same) {
        constexpr int kAhead = 8;
        int t[kAhead], n = 0;
        typename Eight<T>::type x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; j++) {                       // (behind the last one, that again)
            t[j] = same ? 64 * wave + __builtin_ctzll(same) : t[max(j - 1, 0)];
            n += same ? 1 : 0;
            same &= same - 1;
        }
#pragma unroll
        for (int j = 0; j < kAhead; j++) x[j] = read8<T, NARROW>((const T *)a.d_out.data + t[j] * a.d_out.stride, col, a.channels);
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            if (j >= n) break;
            float v[8];
            place8<T, NARROW>(col, a.channels, x[j]);
            widen8<T>(v, x[j]);
            if (l.d.least) draw.apply(v, (uint32_t)t[j]);
#pragma unroll
            for (int k = 0; k < 8; k++) sum[k] += v[k];
        }
    }
    if (wave != first) {
        sums[wave][0][lane] = float4v{sum[0], sum[1], sum[2], sum[3]};
        sums[wave][1][lane] = float4v{sum[4], sum[5], sum[6], sum[7]};
    }
    __syncthreads();
    if (wave != first) return;
    for (int w = first + 1; w < WAVES; w++)
        if (found[w]) {
            const float4v x = sums[w][0][lane], y = sums[w][1][lane];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                sum[k] += x[k];
                sum[4 + k] += y[k];
            }
        }
    put_row(a, row, sum, col);
}

// Sums over runs of sorted places, eight columns a lane.  Rows that lie inside a run are whole; of the row that it begins within and of the
// one that goes on behind it, it leaves a part.  The workgroups behind these fill the other rows, whose stores hide the way of the sums' reads.  WIDE: a run's columns
// take whole waves, which so read rows and places by the scalar unit
template <typename T, bool WIDE, bool NARROW>
__global__ __launch_bounds__(kThreads) void sum_kernel(EmbedLaunch l)
{
    constexpr int kAhead = 8;
    const tessel_embedding &a = l.a;
    if (blockIdx.x >= l.sum_groups) {
        for (int64_t piece = blockIdx.x - l.sum_groups; piece < l.fills; piece += gridDim.x - l.sum_groups) {
            const Piece p(l, piece);
            fill<kThreads>(l, p, [&](int r) { return l.count[((p.row + r) & ((1 << l.shift) - 1)) * l.bins + ((p.row + r) >> l.shift)] != 0; });
        }
        return;
    }
    const int group = blockIdx.x / l.tiles, tile = blockIdx.x % l.tiles;
    int run = group * (kThreads / l.lanes) + threadIdx.x / l.lanes;
    if constexpr (WIDE) run = __builtin_amdgcn_readfirstlane(run);
    const int col = 8 * (tile * l.lanes + threadIdx.x % l.lanes), total = *l.total;
    const int64_t first = (int64_t)run * l.run;
    // eight sorted places at once; behind the last one whatever is there, as some place
    int r[kAhead], t[kAhead];
    const auto look = [&](uint32_t i) {
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            r[j] = l.row[i + j];
            t[j] = (int)min((uint32_t)l.place[i + j], (uint32_t)a.tokens - 1u);
        }
    };
    if (run >= l.runs) return;
    const uint32_t begin = (uint32_t)first, end = (uint32_t)min(first + l.run, (int64_t)total);
    look(begin);
    const int last = l.row[min(first + l.run, a.tokens) - 1], behind = l.row[min(first + l.run, a.tokens - 1)], before = l.row[max(first - 1, (int64_t)0)];
    if (first >= total || col >= a.channels) return;
    const Draw draw(l.d, a.channels, col);
    int row = r[0];
    bool starts = begin == 0 || before != row;                   // (the row's first place is in this run)
    const bool goes_on = first + l.run < total && behind == last;
    float sum[8] = {};
    const auto flush = [&](bool ends) {
        if (starts && ends) {
            put_row(a, row, sum, col);
        } else {
            float4v *to = (float4v *)(l.parts + ((int64_t)run * 2 + (starts ? 1 : 0)) * l.part + col);
            to[0] = float4v{sum[0], sum[1], sum[2], sum[3]};
            to[1] = float4v{sum[4], sum[5], sum[6], sum[7]};
        }
    };
    for (uint32_t i = begin; i < end; i += kAhead) {
        typename Eight<T>::type x[kAhead];
        if (i > begin) look(i);
#pragma unroll
        for (int j = 0; j < kAhead; j++) x[j] = read8<T, NARROW>((const T *)a.d_out.data + t[j] * a.d_out.stride, col, a.channels);
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
            place8<T, NARROW>(col, a.channels, x[j]);
            widen8<T>(v, x[j]);
            if (l.d.least) draw.apply(v, (uint32_t)t[j]);
#pragma unroll
            for (int k = 0; k < 8; k++) sum[k] += v[k];
        }
    }
    flush(!goes_on);
}

// Where a row goes on behind the run that it starts in: the sum of what the runs left of it, four columns a lane.  A workgroup for each run
// and tile of columns; most runs have none.  All that the decision needs is read at once.
__global__ __launch_bounds__(kSortThreads) void join_kernel(EmbedLaunch l, int lanes, int tiles)
{
    __shared__ float4v sums[kSortThreads];
    const tessel_embedding &a = l.a;
    const int run = blockIdx.x / tiles, tile = blockIdx.x % tiles, lane = threadIdx.x & 63, total = *l.total;
    const int64_t first = (int64_t)run * l.run, next = first + l.run, end = a.tokens - 1;
    const int row = l.row[min(next - 1, end)], behind = l.row[min(next, end)], begin = l.row[min(first, end)], before = l.row[max(first - 1, (int64_t)0)];
    int64_t i = next + (int64_t)lane * l.run;
    int more = 0, at = l.row[min(i, end)];
    if (next >= total || behind != row || (begin == row && run > 0 && before == row)) return;
    for (;;) {                                                   // runs that it goes on in
        const uint64_t there = __ballot(i < total && at == row);
        const int n = there == ~0ull ? 64 : __ffsll((unsigned long long)~there) - 1;
        more += n;
        if (n < 64) break;
        i += (int64_t)64 * l.run;
        at = l.row[min(i, end)];
    }
    const int groups = kSortThreads / lanes, group = threadIdx.x / lanes, place = threadIdx.x % lanes, col = 4 * (tile * lanes + place);
    float4v sum = {}, old = {};
    float *to = a.dtable + row * a.dtable_stride + col;
    if (col < a.channels) {
        if (a.accumulate && group == 0) {                        // (under way beside the parts)
#pragma unroll
            for (int j = 0; j < 4; j++) old[j] = to[min(j, a.channels - 1 - col)];
        }
        const float *own = l.parts + ((int64_t)run * 2 + 1) * l.part + col, *others = own + l.part;      // (behind a run's second part, the next one's first)
        if (group == 0) sum = *(const float4v *)own;
#pragma unroll 8
        for (int p = group; p < more; p += groups) sum += *(const float4v *)(others + (int64_t)p * 2 * l.part);
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (group > 0 || col >= a.channels) return;
    for (int g = 1; g < min(groups, more); g++) sum += sums[g * lanes + place];
#pragma unroll
    for (int j = 0; j < 4; j++)
        if (col + j < a.channels) to[j] = old[j] + a.scale * sum[j];
}

int launch_embed(const tessel_embedding &a, const DropLaunch &d, void *stream)
{
    tessel_embedding aa = a;
    DropLaunch dd = d;
    const int rows = span_rows(a.type, a.tokens, a.channels, d, INT32_MAX);
    SpanShape s = span_shape(a.tokens, a.channels, rows);
    void *args[] = {&aa, &dd, &s.lanes};
#define KERNEL(T) (s.wide ? rows == 4 ? (const void *)embed_kernel<T, true, 4> : (const void *)embed_kernel<T, true, 1> \
                          : rows == 4 ? (const void *)embed_kernel<T, false, 4> : (const void *)embed_kernel<T, false, 1>)
    return launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)s.groups), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
}

// Batches that few_kernel takes.  Tokens all different, 1024 channels added to: 256 tokens 3.1 us (13.2 by sort, sums and join), 512 5.2 (13.2), 1024 16.5 (15.2); 4096 channels:
// 256 5.0 (14.8), 512 13.5 (15), 1024 57 (17.7).  One token everywhere: 256 10.3 (13.0), 512 12.4 (13.7), 1024 19 (18.8).
static bool few(const tessel_embedding &a) { return a.tokens <= 256 || (a.tokens <= 512 && a.channels <= 4096); }

static EmbedLaunch embed_launch(const tessel_embedding &a)
{
    EmbedLaunch l = {};
    l.a = a;
    l.shift = 8;
    while (((int64_t)a.rows + (1 << l.shift) - 1) >> l.shift > kMostBins) l.shift++;
    l.bins = (int)(((int64_t)a.rows + (1 << l.shift) - 1) >> l.shift);
    l.lanes = 8;
    while (l.lanes < 256 && 8 * l.lanes < a.channels) l.lanes *= 2;
    l.tiles = (int)(((int64_t)a.channels + 8 * l.lanes - 1) / (8 * l.lanes));
    l.part = ((int64_t)a.channels + 7) / 8 * 8;
    // Places a run: few enough that the runs fill the GPU, and that there are at most 1024 of them, whose parts are read again (8192 tokens of 4096: 32 a run, sums
    // and zeros 164 us and join 8; 16 a run 165 and 11).
    const int64_t threads = a.tokens * (l.part / 8);
    l.run = 8;
    while (l.run < threads >> 17 || (int64_t)l.run * 1024 < a.tokens) l.run *= 2;
    l.runs = (int)((a.tokens + l.run - 1) / l.run);
    l.sum_groups = (uint32_t)((l.runs + kThreads / l.lanes - 1) / (kThreads / l.lanes) * l.tiles);
    l.fill_lanes = 1;
    while (l.fill_lanes < 64 && 4 * (int)l.fill_lanes < a.channels) l.fill_lanes *= 2;
    l.fill_rows = (uint32_t)std::max(1, kFill / a.channels);
    l.fill_pieces = (uint32_t)(((int64_t)a.channels + kFill - 1) / kFill);
    l.fills = a.accumulate ? 0 : (a.rows + (int64_t)l.fill_rows - 1) / l.fill_rows * l.fill_pieces;
    if (few(a)) {
        l.tiles = (int)(((int64_t)a.channels + 511) / 512);
        l.sum_groups = (uint32_t)(a.tokens * l.tiles);
    }
    return l;
}

static size_t whole_chunks(int64_t words) { return (size_t)(words + 3) / 4 * 4; }
static size_t sorted_of(const tessel_embedding &a) { return whole_chunks(a.tokens + 8); }      // (sum_kernel reads eight at once)
static size_t counts_of(const tessel_embedding &a, const EmbedLaunch &l) { return a.accumulate ? 0 : whole_chunks((int64_t)l.bins << l.shift); }

size_t embed_workspace(const tessel_embedding &a)
{
    if (few(a)) return 0;
    const EmbedLaunch l = embed_launch(a);
    return 4 * (2 * sorted_of(a) + 4 + counts_of(a, l) + (size_t)l.runs * 2 * l.part);
}

int launch_embed_backward(const tessel_embedding &a, const DropLaunch &d, void *workspace, void *stream)
{
    EmbedLaunch l = embed_launch(a);
    l.d = d;
    void *args[] = {&l};
    const int64_t groups = l.sum_groups + std::min(l.fills, (int64_t)1 << 20);
    if (few(a)) {
        const int waves = a.tokens <= 256 ? 4 : 8;
#define PICK(T, W) (a.channels < 8 ? (const void *)few_kernel<T, W, true> : (const void *)few_kernel<T, W, false>)
#define KERNEL(T) (waves == 4 ? PICK(T, 4) : PICK(T, 8))
        return groups ? launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)groups), dim3(64 * waves), args, 0, (hipStream_t)stream)) : 0;
#undef KERNEL
#undef PICK
    }
    l.place = (int32_t *)workspace;
    l.row = l.place + sorted_of(a);
    l.total = l.row + sorted_of(a);
    l.count = l.total + 4;
    l.parts = (float *)(l.count + counts_of(a, l));
    const void *sort = a.index_type == TESSEL_I64 ? (const void *)sort_kernel<int64_t> : (const void *)sort_kernel<int32_t>;
    int e = launched(hipLaunchKernel(sort, dim3(1u << l.shift), dim3(kSortThreads), args, 0, (hipStream_t)stream));
#define KERNEL(T) (l.lanes >= 64 ? (const void *)sum_kernel<T, true, false> : (const void *)sum_kernel<T, false, true>)
    if (e == 0 && groups > 0) e = launched(hipLaunchKernel(BY_TYPE(a.type, KERNEL), dim3((unsigned)groups), dim3(kThreads), args, 0, (hipStream_t)stream));
#undef KERNEL
    if (e == 0 && l.runs > 1) {
        int lanes = 16, tiles;
        while (lanes < 256 && 4 * lanes < a.channels) lanes *= 2;
        tiles = (int)(((int64_t)a.channels + 4 * lanes - 1) / (4 * lanes));
        void *more[] = {&l, &lanes, &tiles};
        e = launched(hipLaunchKernel((const void *)join_kernel, dim3((unsigned)(l.runs * tiles)), dim3(kSortThreads), more, 0, (hipStream_t)stream));
    }
    return e;
}

}  // namespace tessel
