// Matrix tiles of the block operators: element types, matrix instructions, layouts in LDS.  (Included by kernel sources only.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tessel {

typedef __bf16   bf16;
typedef _Float16 f16;
typedef float    float4v __attribute__((ext_vector_type(4)));
typedef float    float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Eight values of a type, as one operand of a matrix instruction.
template <typename T> struct Vec8;
template <> struct Vec8<bf16> { typedef bf16 type __attribute__((ext_vector_type(8))); };
template <> struct Vec8<f16> { typedef f16 type __attribute__((ext_vector_type(8))); };

// c += a b, 32 x 16 times 16 x 32.  a: lane holds row lane % 32, columns 8 (lane / 32) + 0..7; b: column lane % 32, rows
// 8 (lane / 32) + 0..7; c: column lane % 32, register i row 8 (i / 4) + 4 (lane / 32) + i % 4.
template <typename T>
__device__ __forceinline__ float16v mma(uint4v a, uint4v b, float16v c)
{
    typedef typename Vec8<T>::type V;
    if constexpr (__is_same(T, bf16))
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}

// two values rounded to the nearest, as one word
template <typename T>
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    typedef T V __attribute__((ext_vector_type(2)));
    V v = {(T)x, (T)y};
    return __builtin_bit_cast(uint32_t, v);
}

// Registers 8 s .. 8 s + 7 of a product's c as the b operand of the next product: the summed index of that operand's
// slot (lane / 32, j) is then 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4, and its a operand is read in the same order.
template <typename T>
__device__ __forceinline__ uint4v operand(const float16v &c, int s)
{
    uint4v r;
#pragma unroll
    for (int j = 0; j < 4; j++) r[j] = pack2<T>(c[8 * s + 2 * j], c[8 * s + 2 * j + 1]);
    return r;
}

// A tile of rows of W values (2 bytes each) in LDS (its start: a multiple of 256 bytes), rows packed, chunks of 16 bytes of a row swapped so that both ways
// of reading touch all banks: 16 rows at one column (row operands), and 4 rows x 32 columns (transposing reads).
template <int W>
__device__ __forceinline__ int chunk_at(int row, int chunk)          // in chunks of 16 bytes
{
    if constexpr (W == 128) return row * 16 + (chunk ^ ((row & 3) << 2 | (row >> 2 & 3)));
    else return row * 8 + (chunk ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3)));
}

typedef __attribute__((address_space(3))) uint4v lds_uint4v;
typedef __attribute__((address_space(3))) const uint4v lds_tile;

// Where a lane reads operands from a tile in LDS: two byte addresses, from which those of all operands come by one exclusive or and a
// constant offset (the swaps of chunk_at are exclusive ors too, and tiles start at multiples of 256 bytes).  hold() keeps the
// compiler from working the addresses of a loop out before it and keeping them all in registers.
template <int W>
struct Reader {
    uint32_t r, c;
    __device__ __forceinline__ Reader()
    {
        const int lane = threadIdx.x & 63, i = lane & 15, row = 4 * (lane >> 5) + (i >> 2);
        r = 16 * chunk_at<W>(lane & 31, lane >> 5);
        c = 16 * chunk_at<W>(row, 2 * (lane >> 4 & 1) + (i >> 1 & 1)) + 8 * (i & 1);
    }
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(r), "+v"(c)); }
    // a operand of the tile's rows row .. row + 31 (row: a multiple of 16), columns 16 s .. 16 s + 15; also a b operand, for a tile that
    // holds columns as rows
    __device__ __forceinline__ uint4v rows(const lds_tile *tile, int row, int s) const
    {
        return *(const lds_tile *)((uint32_t)(uintptr_t)tile + (r ^ (32 * s)) + row * 2 * W);
    }
};

// Column operands of one step of sixteen rows for all W / 32 blocks: a operands whose rows are 32 columns of the tile and whose summed index are
// its rows, in the order of operand().  Each is two transposing reads, of which a group of 16 lanes takes 4 rows x 16 columns, all in one piece
// that ends when they have arrived.  (Where the compiler places a transposing read itself, it first waits for every copy to LDS that is on its
// way.)  `at`: the addresses of the blocks' two halves in the tile, `OFFSET`: the step's distance from its start.
__device__ __forceinline__ uint4v join(uint64_t lo, uint64_t hi)
{
    typedef uint64_t V __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint4v, V{lo, hi});
}
template <int W>
__device__ __forceinline__ void column_addresses(uint32_t *at, const lds_tile *tile, const Reader<W> &r)
{
#pragma unroll
    for (int b = 0; b < W / 16; b++) at[b] = (uint32_t)(uintptr_t)tile + (r.c ^ (32 * b));
}
template <int OFFSET>
__device__ __forceinline__ void read_columns(uint4v (&f)[4], const uint32_t (&at)[8])
{
    uint64_t r[8];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%16\n\tds_read_b64_tr_b16 %1, %9 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %2, %10 offset:%16\n\tds_read_b64_tr_b16 %3, %11 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %4, %12 offset:%16\n\tds_read_b64_tr_b16 %5, %13 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %6, %14 offset:%16\n\tds_read_b64_tr_b16 %7, %15 offset:%17\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]), "v"(at[7]), "n"(OFFSET), "n"(OFFSET + 8 * 256)
                 : "memory");
#pragma unroll
    for (int b = 0; b < 4; b++) f[b] = join(r[2 * b], r[2 * b + 1]);
}
template <int OFFSET>
__device__ __forceinline__ void read_columns(uint4v (&f)[2], const uint32_t (&at)[4])
{
    uint64_t r[4];
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %1, %5 offset:%9\n\t"
                 "ds_read_b64_tr_b16 %2, %6 offset:%8\n\tds_read_b64_tr_b16 %3, %7 offset:%9\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(OFFSET), "n"(OFFSET + 8 * 128)
                 : "memory");
#pragma unroll
    for (int b = 0; b < 2; b++) f[b] = join(r[2 * b], r[2 * b + 1]);
}

// a loop whose counter is a constant in each turn: body(constant<0>) .. body(constant<N - 1>)
template <int I> struct constant {
    static constexpr int value = I;
};
template <int N, int I = 0, typename F>
__device__ __forceinline__ void unrolled(F &&body)
{
    if constexpr (I < N) {
        body(constant<I>{});
        unrolled<N, I + 1>(body);
    }
}

typedef __attribute__((address_space(1))) const uint4v global_uint4v;

// A tile of 64 rows x W on its way from memory straight to LDS by all threads of a workgroup, without passing registers: a wave's
// instruction fills 1 KB of LDS from its start on, so the lanes pick the chunks of their rows in the order of chunk_at.  Rows from
// `rows` on and columns from dim on are left as they are in LDS.
template <typename T, int W, int THREADS>
struct Copy {
    static constexpr int kChunks = W / 8, kRows = THREADS / kChunks, kPer = 64 / kRows;
    static_assert(kRows % 16 == 0, "the order of chunks repeats after 16 rows");
    __device__ __forceinline__ static void start(uint4v *tile, const T *base, int64_t stride, int rows, int dim)
    {
        const int r = threadIdx.x / kChunks, c = (threadIdx.x % kChunks) ^ (chunk_at<W>(r, 0) % kChunks);
        const T *p = base + r * stride + 8 * c;
        lds_uint4v *to = (lds_uint4v *)(tile + __builtin_amdgcn_readfirstlane(threadIdx.x & ~63));
        if (rows >= 64 && dim == W) {
#pragma unroll
            for (int i = 0; i < kPer; i++) __builtin_amdgcn_global_load_lds((global_uint4v *)(p + i * kRows * stride), to + i * THREADS, 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; i++)
                if (r + i * kRows < rows && 8 * c < dim)
                    __builtin_amdgcn_global_load_lds((global_uint4v *)(p + i * kRows * stride), to + i * THREADS, 16, 0, 0);
        }
    }
};

// Waits until this wave's copies are in LDS, then for the other waves.  (A barrier alone waits for no copy: what goes from memory
// to LDS counts as a load from memory.)
__device__ __forceinline__ void copies_arrive()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// sum and maximum of a value and that of the same column in the other half-wave
__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

}  // namespace tessel
