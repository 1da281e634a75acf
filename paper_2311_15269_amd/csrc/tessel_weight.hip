// Gradient of a product's weights from an input kept in 8 bits: dw[n][c] = sum_t dy[t][n] x[t][c] (include/tessel_block_ops.h).
//
// A workgroup takes a tile of dw and goes over the tokens 64 at a time; each wave has 64 columns (c) of it and 32 MB rows (n).  The summed
// index runs along the rows of both inputs, so both operands come out of LDS by transposing reads.  The checkpoint is turned into
// numbers of the matrix instruction's type on its way to LDS, which is exact.  Few tiles: the tokens are split over several
// workgroups, whose sums a second kernel adds in the order of their numbers.
//
// Bound by the matrix instructions, and with them by the clock that they leave: 4096 x 4096 from 8192 tokens of bf16 in 248 us, 1110 TF/s (a
// library product of 16-bit inputs of that shape takes 230 to 285 us, the input first written out in 16 bits not counted).  A wave's
// 128 x 64 reads six operands from LDS for eight products, so that LDS is not the bound.  Small ones are bound by the time from a tile's
// reads to its use and by the parts' traffic: 1001 x 715 from 1999 tokens in 23.5 us, 5 of them the second kernel.
#include "tessel_rows.h"

namespace tessel {

constexpr int kSteps = 64;       // tokens at a time
constexpr int kPanel = 128;      // columns of a panel in LDS
constexpr int kPanelSize = kSteps * kPanel / 8;

struct WeightLaunch {
    tessel_weight_grad a;
    float  *parts;               // [splits][outputs][channels], or NULL: one split, straight to dw
    int     splits;
    int64_t per;                 // tokens a split, a multiple of kSteps
    int     tiles_c;
};

// What dy looks like decides how it comes to LDS.
//   kStraight  rows of whole chunks of 16 bytes: from memory to LDS without passing registers, three buffers.  Copies start two tiles ahead; the
//              checkpoint's bytes pass registers, and the compiler's wait before it writes them to LDS is for all reads, so that it ends the
//              next tile's copies too: in the large tiles every time, in the small ones every other time
//   kUneven    other rows of eight outputs or more, through registers: a chunk that would pass the row's end starts eight before it
//   kNarrow    fewer outputs, value by value
// (No load stands in a branch: the compiler would wait for it where the branch ends.)
enum { kStraight, kUneven, kNarrow };

// the output that a lane's chunk at output n starts with
template <int HOW>
__device__ __forceinline__ int chunk_start(int n, int outputs) { return HOW == kNarrow ? n : min(n, outputs - 8); }

// 64 tokens x COLUMNS of dy through registers.  Rows behind the tokens repeat the last one and are put as zeros.
template <typename T, int COLUMNS, int THREADS, int HOW>
struct DyStage {
    static constexpr int kChunks = COLUMNS / 8, kPer = kSteps * kChunks / THREADS, kRows = THREADS / kChunks;
    typename Eight<T>::type v[kPer];
    __device__ __forceinline__ void fetch(const tessel_weight_grad &a, int64_t t0, int64_t end, int n0, int thread)
    {
        const int r = thread / kChunks, col = chunk_start<HOW>(n0 + 8 * (thread % kChunks), a.outputs);
        const T *p = (const T *)a.dy.data + t0 * a.dy.stride;
        const uint32_t stride = (uint32_t)a.dy.stride, last = (uint32_t)min((int64_t)kSteps, end - t0) - 1;
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            const uint32_t row = min((uint32_t)(r + i * kRows), last) * stride;
            if constexpr (HOW == kNarrow) {
#pragma unroll
                for (int j = 0; j < 8; j++) v[i][j] = p[row + (uint32_t)min(col + j, a.outputs - 1)];
            } else {
                v[i] = *(const typename Eight<T>::type *)(p + (row + (uint32_t)col));
            }
        }
    }
    __device__ __forceinline__ void put(uint4v *tile, int rows, int thread) const
    {
        const int r = thread / kChunks, c = thread % kChunks;
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            uint4v w = __builtin_bit_cast(uint4v, v[i]);
            if (r + i * kRows >= rows) w = uint4v{0, 0, 0, 0};
            tile[c / 16 * kPanelSize + chunk_at<kPanel>(r + i * kRows, c % 16)] = w;
        }
    }
};

// The same from memory straight to LDS.  Columns behind the outputs and rows behind the tokens repeat the last ones; the rows are
// overwritten with zeros (clear), the columns' sums are not stored.
template <typename T, int COLUMNS, int THREADS>
struct DyCopy {
    static constexpr int kChunks = COLUMNS / 8, kPer = kSteps * kChunks / THREADS;
    static constexpr int kRows = THREADS / 16, kEach = kSteps / kRows;         // a panel at a time: rows an instruction, instructions
    static_assert(kRows % 16 == 0 && kEach * (COLUMNS / kPanel) == kPer, "the order of chunks repeats after 16 rows");
    __device__ __forceinline__ static void start(uint4v *tile, const tessel_weight_grad &a, int64_t t0, int64_t end, int n0, int thread)
    {
        const int r = thread / 16, c = (thread % 16) ^ (chunk_at<kPanel>(r, 0) % 16);
        const T *p = (const T *)a.dy.data + t0 * a.dy.stride;
        const uint32_t stride = (uint32_t)a.dy.stride, last = (uint32_t)min((int64_t)kSteps, end - t0) - 1;
        lds_uint4v *to = (lds_uint4v *)(tile + __builtin_amdgcn_readfirstlane(thread & ~63));
#pragma unroll
        for (int b = 0; b < COLUMNS / kPanel; b++) {
            const uint32_t col = min(n0 + b * kPanel + 8 * c, a.outputs - 8);
#pragma unroll
            for (int i = 0; i < kEach; i++)
                __builtin_amdgcn_global_load_lds((global_uint4v *)(p + (min((uint32_t)(r + i * kRows), last) * stride + col)), to + b * kPanelSize + i * THREADS, 16, 0, 0);
        }
    }
    __device__ __forceinline__ static void clear(uint4v *tile, int rows, int thread)
    {
        for (int k = thread; k < (kSteps - rows) * kChunks; k += THREADS)
            tile[k / (16 * (kSteps - rows)) * kPanelSize + (rows + k / 16 % (kSteps - rows)) * 16 + k % 16] = uint4v{0, 0, 0, 0};
    }
};

// 64 tokens x COLUMNS of a checkpoint through registers, sixteen values a lane.  Columns behind the channels repeat others.
template <typename T, int COLUMNS, int THREADS>
struct HeldStage {
    static constexpr int kChunks = COLUMNS / 16, kPer = kSteps * kChunks / THREADS, kRows = THREADS / kChunks;
    uint4v   v[kPer];
    uint32_t e[kPer];
    __device__ __forceinline__ void fetch(const tessel_weight_grad &a, int64_t t0, int64_t end, int c0, int thread)
    {
        const int r = thread / kChunks;
        const uint32_t col = min(c0 + 16 * (thread % kChunks), (a.x.channels - 1) & ~15);   // (behind the channels, values to the end of the group)
        const int8_t *p = a.x.values + t0 * a.x.value_stride;
        const uint8_t *q = a.x.exponents + t0 * a.x.exponent_stride;
        const uint32_t last = (uint32_t)min((int64_t)kSteps, end - t0) - 1;
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            const uint32_t row = min((uint32_t)(r + i * kRows), last);
            v[i] = *(const uint4v *)(p + (row * (uint32_t)a.x.value_stride + col));
            e[i] = q[row * (uint32_t)a.x.exponent_stride + col / kGroup];
        }
    }
    // rows: of which tokens there are
    __device__ __forceinline__ void put(uint4v *tile, int rows, int i, int thread) const
    {
        const int r = thread / kChunks + i * kRows, c = 2 * (thread % kChunks);
        uint4v bytes = v[i];
        uint32_t exponent = e[i];
        asm volatile("" : "+v"(bytes), "+v"(exponent));          // (or the compiler takes the bytes apart where it reads them, and waits for them there)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float f[8];
            held8(f, make_uint2(bytes[2 * h], bytes[2 * h + 1]), exponent);
            uint4v w;
#pragma unroll
            for (int j = 0; j < 4; j++) w[j] = pack2<T>(f[2 * j], f[2 * j + 1]);
            if (r >= rows) w = uint4v{0, 0, 0, 0};
            tile[c / 16 * kPanelSize + chunk_at<kPanel>(r, (c + h) % 16)] = w;
        }
    }
};

// The operands of one step of sixteen tokens, MB of rows and two of columns, by transposing reads from LDS in one piece that ends when all
// have arrived.  (The compiler, where it places such a read itself, first waits for every copy to LDS that is on its way.)
template <int S>
__device__ __forceinline__ void read_step(uint4v (&f)[4], uint4v (&g)[2], const uint32_t (&x)[8], const uint32_t (&y)[4])
{
    uint64_t r[12];
    asm volatile("ds_read_b64_tr_b16 %0, %12 offset:%24\n\tds_read_b64_tr_b16 %1, %13 offset:%25\n\t"
                 "ds_read_b64_tr_b16 %8, %20 offset:%24\n\tds_read_b64_tr_b16 %9, %21 offset:%25\n\t"
                 "ds_read_b64_tr_b16 %2, %14 offset:%24\n\tds_read_b64_tr_b16 %3, %15 offset:%25\n\t"
                 "ds_read_b64_tr_b16 %10, %22 offset:%24\n\tds_read_b64_tr_b16 %11, %23 offset:%25\n\t"
                 "ds_read_b64_tr_b16 %4, %16 offset:%24\n\tds_read_b64_tr_b16 %5, %17 offset:%25\n\t"
                 "ds_read_b64_tr_b16 %6, %18 offset:%24\n\tds_read_b64_tr_b16 %7, %19 offset:%25\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]),
                   "=&v"(r[10]), "=&v"(r[11])
                 : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(x[4]), "v"(x[5]), "v"(x[6]), "v"(x[7]), "v"(y[0]), "v"(y[1]), "v"(y[2]), "v"(y[3]),
                   "n"(S * 16 * 2 * kPanel), "n"(S * 16 * 2 * kPanel + 8 * 2 * kPanel)
                 : "memory");
#pragma unroll
    for (int b = 0; b < 4; b++) f[b] = join(r[2 * b], r[2 * b + 1]);
#pragma unroll
    for (int b = 0; b < 2; b++) g[b] = join(r[8 + 2 * b], r[9 + 2 * b]);
}
template <int S>
__device__ __forceinline__ void read_step(uint4v (&f)[2], uint4v (&g)[2], const uint32_t (&x)[4], const uint32_t (&y)[4])
{
    uint64_t r[8];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%16\n\tds_read_b64_tr_b16 %1, %9 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %4, %12 offset:%16\n\tds_read_b64_tr_b16 %5, %13 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %2, %10 offset:%16\n\tds_read_b64_tr_b16 %3, %11 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %6, %14 offset:%16\n\tds_read_b64_tr_b16 %7, %15 offset:%17\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                 : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(y[0]), "v"(y[1]), "v"(y[2]), "v"(y[3]),
                   "n"(S * 16 * 2 * kPanel), "n"(S * 16 * 2 * kPanel + 8 * 2 * kPanel)
                 : "memory");
#pragma unroll
    for (int b = 0; b < 2; b++) f[b] = join(r[2 * b], r[2 * b + 1]);
#pragma unroll
    for (int b = 0; b < 2; b++) g[b] = join(r[4 + 2 * b], r[5 + 2 * b]);
}

// A barrier behind this wave's LDS writes.  (The library's waits for all loads from memory too, also those that belong to later tiles.)
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// nothing is moved across, by any pass of the compiler
__device__ __forceinline__ void in_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Reads from memory that a wait further on counts on: it lets the last so many be under way, so one that the compiler merged with another, left out
// or moved behind the end would let one of the copies before them be, too.  The build counts them in the listing, between these two marks.
__device__ __forceinline__ void counted_reads()
{
    in_order();
    asm volatile("; counted reads begin" ::: "memory");
}
template <int READS>
__device__ __forceinline__ void counted_reads_end()
{
    asm volatile("; counted reads end %0" ::"n"(READS) : "memory");
    in_order();
}
template <int READS>
__device__ __forceinline__ void wait_for_all_but()
{
    asm volatile("s_waitcnt vmcnt(%0) ; counted" ::"n"(READS) : "memory");
}

// WN x WC waves, 32 MB x 64 of dw each, GROUPS times, each group for its share of the workgroup's tokens (two, where tiles are small: with half as many
// parts in memory as two workgroups would leave).  DEPTH: tiles on their way in registers
template <typename T, int WN, int WC, int MB, int HOW, int GROUPS, int DEPTH>
__global__ __launch_bounds__(64 * WN * WC * GROUPS, 2) void weight_kernel(WeightLaunch l)
{
    constexpr int kThreads = 64 * WN * WC, kRows = WN * MB * 32, kColumns = WC * 64, kBuffers = HOW == kStraight ? 3 : 2;
    static_assert(kRows % kPanel == 0 && kColumns % kPanel == 0, "whole panels");
    typedef DyCopy<T, kRows, kThreads> Copy;
    __shared__ __attribute__((aligned(256))) uint4v all_rows[GROUPS][kBuffers][kSteps * kRows / 8], all_columns[GROUPS][2][kSteps * kColumns / 8];
    const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads), thread = threadIdx.x % kThreads;
    uint4v (*const rows)[kSteps * kRows / 8] = all_rows[group], (*const columns)[kSteps * kColumns / 8] = all_columns[group];
    const tessel_weight_grad &a = l.a;
    // workgroups go to the eight L2 caches in turn: each cache gets neighbouring tiles, which share their inputs
    const int all = gridDim.x, per = all / 8, more = all % 8, x = blockIdx.x % 8;
    const int place = x * per + min(x, more) + blockIdx.x / 8;
    const int n0 = place / l.tiles_c * kRows, c0 = place % l.tiles_c * kColumns;
    // the first group's share has as many steps as any other's: all go through its barriers
    const int64_t from = blockIdx.y * l.per, to = min(from + l.per, a.x.tokens), share = ((to - from + kSteps - 1) / kSteps + GROUPS - 1) / GROUPS;
    const int64_t begin = min(from + group * share * kSteps, to), end = min(begin + share * kSteps, to);
    const int wave = thread >> 6, lane = threadIdx.x & 63, half = lane >> 5;
    const int wn = wave / WC * MB, wc = wave % WC * 2;           // in blocks of 32
    float16v acc[MB][2] = {};
    if (from < to) {
        const Reader<kPanel> at;
        uint32_t fx[2 * MB], gy[4];                              // operands' addresses: blocks of 32, both halves of their eight tokens
#pragma unroll
        for (int b = 0; b < MB; b++)
#pragma unroll
            for (int h = 0; h < 2; h++) fx[2 * b + h] = (uint32_t)(uintptr_t)(lds_tile *)rows[0] + (wn + b) / 4 * kPanelSize * 16 + (at.c ^ (64 * ((wn + b) % 4) + 32 * h));
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int h = 0; h < 2; h++) gy[2 * b + h] = (uint32_t)(uintptr_t)(lds_tile *)columns[0] + wc / 4 * kPanelSize * 16 + (at.c ^ (64 * (wc % 4 + b) + 32 * h));
        HeldStage<T, kColumns, kThreads> hs[DEPTH];
        DyStage<T, HOW == kStraight ? 8 : kRows, HOW == kStraight ? 8 : kThreads, HOW> ds[DEPTH];
        constexpr int kHeld = hs[0].kPer;
        const int64_t tiles = (end - begin + kSteps - 1) / kSteps;
        auto left = [&](int64_t n) { return (int)min((int64_t)kSteps, end - begin - n * kSteps); };
        // tile n to stage `stage` of the registers, the rest of it from memory to LDS, and from the registers to LDS
        auto fetch = [&](int stage, int64_t n) {
            if constexpr (HOW == kStraight) counted_reads();
            hs[stage].fetch(a, begin + n * kSteps, end, c0, thread);
            if constexpr (HOW == kStraight) counted_reads_end<2 * kHeld>();
            else ds[stage].fetch(a, begin + n * kSteps, end, n0, thread);
        };
        auto copy = [&](int64_t n, int to) {
            if constexpr (HOW == kStraight) {
                counted_reads();
                Copy::start(rows[to], a, begin + n * kSteps, end, n0, thread);
                counted_reads_end<Copy::kPer>();
            }
        };
        auto put = [&](int stage, int64_t n) {
#pragma unroll
            for (int i = 0; i < kHeld; i++) hs[stage].put(columns[n & 1], left(n), i, thread);
            if constexpr (HOW != kStraight) ds[stage].put(rows[n & 1], left(n), thread);
        };
        // the first tiles, in this order, on which the waits below count: behind a tile's copies come one tile of the checkpoint and the next
        // tile's copies
        auto start = [&](auto more) {
            constexpr bool MORE = decltype(more)::value != 0;
            fetch(0, 0);
            if (DEPTH == 2 && (MORE || tiles > 1)) fetch(1, 1);
            in_order();
            copy(0, 0);
            in_order();
            put(0, 0);
            in_order();
            if (MORE || tiles > DEPTH) fetch(0, DEPTH);
            in_order();
            if (MORE || tiles > 1) copy(1, 1);
            in_order();
        };
        const int64_t short_one = (to - from) % kSteps ? ((to - from) / kSteps) % share : -1;       // the step of the tile that is not whole
        int buffer = 0;
        // One tile.  MORE: all that is to be read behind it is there, so that no read stands in a branch (behind which the compiler would wait for more than
        // it has to)
        auto tile = [&](auto stage, auto more, int64_t n) {
            constexpr int kNext = (decltype(stage)::value + 1) % DEPTH;
            constexpr bool MORE = decltype(more)::value != 0;
            if constexpr (HOW == kStraight) {
                if (MORE || n + DEPTH < tiles) wait_for_all_but<Copy::kPer + 2 * kHeld>();
                else if (DEPTH == 2 && n + 1 < tiles) wait_for_all_but<Copy::kPer>();
                else wait_for_all_but<0>();
                if (!MORE && n == short_one) {
                    lds_barrier();                               // (all waves' copies, before zeros go over them)
                    if (n < tiles) Copy::clear(rows[buffer], left(n), thread);
                }
            }
            lds_barrier();                                       // (this tile is there, and all are done with the one before)
            if (!MORE && GROUPS > 1 && n >= tiles) return;
            uint32_t fa[2 * MB], ga[4];
#pragma unroll
            for (int b = 0; b < 2 * MB; b++) fa[b] = fx[b] + buffer * (kSteps * kRows * 2);
#pragma unroll
            for (int b = 0; b < 4; b++) ga[b] = gy[b] + (uint32_t)(n & 1) * (kSteps * kColumns * 2);
            auto step = [&](auto s) {
                uint4v f[MB], g[2];
                read_step<decltype(s)::value>(f, g, fa, ga);
#pragma unroll
                for (int i = 0; i < MB; i++)
#pragma unroll
                    for (int j = 0; j < 2; j++) acc[i][j] = mma<T>(f[i], g[j], acc[i][j]);
            };
            step(constant<0>{});
            step(constant<1>{});
            if (MORE || n + 1 < tiles) put(kNext, n + 1);
            in_order();
            if (MORE || n + 1 + DEPTH < tiles) fetch(kNext, n + 1 + DEPTH);
            in_order();
            if (MORE || n + 2 < tiles) copy(n + 2, buffer >= 1 ? buffer - 1 : 2);
            in_order();
            step(constant<2>{});
            step(constant<3>{});
            buffer = buffer == kBuffers - 1 ? 0 : buffer + 1;
        };
        int64_t n = 0;
        if (tiles > 2 * DEPTH) {
            start(constant<1>{});
            // (whole tiles alone: the short one is the last of all)
            for (; n + 2 * DEPTH < tiles; n += DEPTH) unrolled<DEPTH>([&](auto c) { tile(c, constant<1>{}, n + decltype(c)::value); });
        } else if (tiles > 0) {
            start(constant<0>{});
        }
        for (; n < share; n += DEPTH)
            unrolled<DEPTH>([&](auto c) {
                if (n + decltype(c)::value < share) tile(c, constant<0>{}, n + decltype(c)::value);
            });
    }
    if constexpr (GROUPS > 1) {
        static_assert(GROUPS == 2 && sizeof(all_rows) >= sizeof(acc) * kThreads, "one group's sums");
        float4v *sums = (float4v *)all_rows + thread;
        __syncthreads();
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < MB * 8; i++) {
                const float16v &c = acc[i / 8][i / 4 % 2];
                sums[i * kThreads] = float4v{c[4 * (i % 4)], c[4 * (i % 4) + 1], c[4 * (i % 4) + 2], c[4 * (i % 4) + 3]};
            }
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int i = 0; i < MB * 8; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i / 8][i / 4 % 2][4 * (i % 4) + j] += sums[i * kThreads][j];
    }
    float *out = l.parts ? l.parts + (int64_t)blockIdx.y * a.outputs * a.x.channels : a.dw;
    const int64_t stride = l.parts ? a.x.channels : a.dw_stride;
    const bool add = !l.parts && a.accumulate;
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const int c = c0 + 32 * (wc + j) + (lane & 31);
        if (c >= a.x.channels) continue;
#pragma unroll
        for (int i = 0; i < MB; i++) {
            float *p[16];
            bool there[16];
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const int chunk = n0 + 32 * (wn + i) + 8 * (r / 4), n = chunk_start<HOW>(chunk, a.outputs) + 4 * half + r % 4;
                there[r] = n < a.outputs && n >= chunk;          // (what a shifted chunk holds of the one before is stored there)
                p[r] = out + (there[r] ? n * stride : 0) + c;
            }
            if (add) {
                float v[16];
#pragma unroll
                for (int r = 0; r < 16; r++) v[r] = *p[r];       // (all sixteen on their way at once; the first row's where there is none)
#pragma unroll
                for (int r = 0; r < 16; r++) acc[i][j][r] += v[r];
            }
#pragma unroll
            for (int r = 0; r < 16; r++)
                if (there[r]) *p[r] = acc[i][j][r];
        }
    }
}

// four values a lane
__global__ __launch_bounds__(256) void weight_sum_kernel(WeightLaunch l)
{
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
    const tessel_weight_grad &a = l.a;
    const int64_t size = (int64_t)a.outputs * a.x.channels, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size) return;
    const int64_t row = i / a.x.channels, col = i - row * a.x.channels;
    float *p = a.dw + row * a.dw_stride + col;
    if (col + 4 <= a.x.channels) {
        V sum = {};
        if (a.accumulate) sum = *(const V *)p;
#pragma unroll 4
        for (int s = 0; s < l.splits; s++) sum += *(const V *)(l.parts + s * size + i);
        *(V *)p = sum;
    } else {
        for (int64_t k = i; k < min(i + 4, size); k++) {
            p = a.dw + k / a.x.channels * a.dw_stride + k % a.x.channels;
            float sum = a.accumulate ? *p : 0.0f;
            for (int s = 0; s < l.splits; s++) sum += l.parts[s * size + k];
            *p = sum;
        }
    }
}

struct WeightShape {
    int     tile;                // rows and columns of dw a workgroup takes
    int64_t tiles;
    int     splits;
};
static WeightShape shape_of(const tessel_weight_grad &a)
{
    auto tiles_of = [&](int64_t n) { return ((a.outputs + n - 1) / n) * ((a.x.channels + n - 1) / n); };
    // Large tiles read LDS less for each product, small ones fill the compute units with less splitting.  Large where more than 128 of them fill the units
    // as they are (1024 tokens, 4096 x 2400: 42 us, small 52), or where the splits that do keep some 1300 tokens (8192 tokens, 2048 x 2048: 104, small 108; 4096
    // tokens, 3500 x 1500: 78, small 93; but 1024 tokens, 4096 x 2048: 45, small 36; 2048 tokens, 2048 x 2048: 45, small 30).
    WeightShape s = {256, tiles_of(256), 1};
    if (a.outputs < 8 || (s.tiles <= 128 && a.x.tokens * s.tiles < 1280 * 256)) s = {128, tiles_of(128), 1};
    // splits of the tokens: until 256 workgroups are there, as many as leave a group more than 128 tokens on average (their last ones, in whole
    // steps, may be shorter: 513 tokens by small tiles are 320 and 193, those of two groups 128 and 65)
    const int64_t least = s.tile == 256 ? 256 : 512, most = (a.x.tokens + least - 1) / least, want = 256 / s.tiles, n = want < most ? want : most;
    s.splits = n < 1 ? 1 : (int)n;
    return s;
}

int64_t weight_tiles(const tessel_weight_grad &a) { return shape_of(a).tiles; }
int weight_parts(const tessel_weight_grad &a) { return shape_of(a).splits; }

int launch_weight_gradient(const tessel_weight_grad &a, float *parts, void *stream)
{
    const WeightShape s = shape_of(a);
    WeightLaunch l = {a, nullptr, s.splits, 0, (int)(((int64_t)a.x.channels + s.tile - 1) / s.tile)};
    l.per = ((a.x.tokens + l.splits - 1) / l.splits + kSteps - 1) / kSteps * kSteps;
    if (l.splits > 1) l.parts = parts;
    void *args[] = {&l};
    const bool large = s.tile == 256, straight = a.outputs % 8 == 0 && a.dy.stride % 8 == 0 && (uintptr_t)a.dy.data % 16 == 0;
#define KERNEL(T) (a.outputs < 8 ? (const void *)weight_kernel<T, 2, 2, 2, kNarrow, 2, 1> \
                   : large ? (straight ? (const void *)weight_kernel<T, 2, 4, 4, kStraight, 1, 1> : (const void *)weight_kernel<T, 2, 4, 4, kUneven, 1, 1>) \
                           : (straight ? (const void *)weight_kernel<T, 2, 2, 2, kStraight, 2, 2> : (const void *)weight_kernel<T, 2, 2, 2, kUneven, 2, 2>))
    const void *kernel = a.x.type == TESSEL_BF16 ? KERNEL(bf16) : KERNEL(f16);
#undef KERNEL
    int e = launched(hipLaunchKernel(kernel, dim3((unsigned)s.tiles, (unsigned)l.splits), dim3(kWeightThreads), args, 0, (hipStream_t)stream));
    if (e == 0 && l.parts)
        e = launched(hipLaunchKernel((const void *)weight_sum_kernel, dim3((unsigned)(((int64_t)a.outputs * a.x.channels + 1023) / 1024)), dim3(256), args, 0, (hipStream_t)stream));
    return e;
}

}  // namespace tessel
