// Rows of values of the three element types, eight at a time, and activation checkpoints.  (Included by kernel sources only.)
#pragma once
#include "tessel_block.h"
#include "tessel_tile.h"

namespace tessel {

constexpr int kGroup = TESSEL_CHECKPOINT_GROUP;

// Eight neighbouring values.  Rows of an odd number of channels start anywhere, so the loads and stores ask for no more than the
// element's alignment (the memory path takes 16 bytes at any address).
template <typename T> struct Eight {
    typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// values col .. col + 7 of a row of `channels`, zeros behind its end, as they are.  The end of a row in pieces of four, two and one.
template <typename T>
__device__ __forceinline__ typename Eight<T>::type raw8(const T *row, int col, int channels)
{
    typedef T V4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef T V2 __attribute__((ext_vector_type(2), aligned(sizeof(T))));
    if (col + 8 <= channels) return *(const typename Eight<T>::type *)(row + col);
    typename Eight<T>::type v = {};
    const int n = channels - col;
    if (n <= 0) return v;
    V4 x = {};
    V2 y = {};
    T z = (T)0.0f;
    if (n & 4) x = *(const V4 *)(row + col);
    if (n & 2) y = *(const V2 *)(row + col + (n & 4));
    if (n & 1) z = row[col + (n & 6)];
    const V2 last = (n & 2) ? y : V2{z, (T)0.0f}, after = (n & 2) ? V2{z, (T)0.0f} : V2{(T)0.0f, (T)0.0f};
    if (n & 4) {
        v[0] = x[0], v[1] = x[1], v[2] = x[2], v[3] = x[3];
        v[4] = last[0], v[5] = last[1], v[6] = after[0];
    } else {
        v[0] = last[0], v[1] = last[1], v[2] = after[0];
    }
    return v;
}

// the same in 32 bits
template <typename T>
__device__ __forceinline__ void load8(float *v, const T *row, int col, int channels)
{
    const typename Eight<T>::type w = raw8<T>(row, col, channels);
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = (float)w[j];
}

// The same without a branch around a read, where the compiler would wait for it: take8 reads, settle8 puts the values in their places, several
// chunks of the same columns at once and behind all reads.  What would pass the row's end is read from eight values before it and moved
// up.  Rows of fewer than eight, where the caller may have such (NARROW): value by value.
template <typename T, bool NARROW>
__device__ __forceinline__ typename Eight<T>::type take8(const T *row, int col, int channels)
{
    if (NARROW && channels < 8) {
        typename Eight<T>::type v;
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = row[min(j, channels - 1)];
        return v;
    }
    return *(const typename Eight<T>::type *)(row + min(col, channels - 8));
}
template <typename T, bool NARROW, typename... V>
__device__ __forceinline__ void settle8(int col, int channels, V &...v)
{
    typedef uint32_t Words __attribute__((ext_vector_type(2 * sizeof(T))));
    constexpr int N = 2 * sizeof(T), kWord = 4 / sizeof(T);
    if (channels & 7) {
        const int by = NARROW && channels < 8 ? (col < channels ? 0 : 8) : col - min(col, channels - 8);
        const auto move = [by](typename Eight<T>::type &x) {
            Words w = __builtin_bit_cast(Words, x);
#pragma unroll
            for (int step = 4; step >= kWord; step /= 2)
#pragma unroll
                for (int j = 0; j < N; j++) w[j] = (by & step) ? (j + step / kWord < N ? w[j + step / kWord] : 0u) : w[j];
            if constexpr (kWord == 2) {
#pragma unroll
                for (int j = 0; j < N; j++) w[j] = (by & 1) ? __builtin_amdgcn_alignbit(j + 1 < N ? w[j + 1] : 0u, w[j], 16) : w[j];
            }
            x = __builtin_bit_cast(typename Eight<T>::type, w);
        };
        (move(v), ...);
    }
    // (a branch where waves have whole chunks; in 32 bits, where its copies cost registers that there are not, without it)
    if (sizeof(T) == 4 || __any(col >= channels || (NARROW && channels < 8))) {
        const auto end = [&](typename Eight<T>::type &x) {
            if (NARROW && channels < 8) {
#pragma unroll
                for (int j = 0; j < 8; j++) x[j] = j < channels ? x[j] : (T)0.0f;
            }
            Words w = __builtin_bit_cast(Words, x);
#pragma unroll
            for (int j = 0; j < N; j++) w[j] = col < channels ? w[j] : 0u;
            x = __builtin_bit_cast(typename Eight<T>::type, w);
        };
        (end(v), ...);
    }
}

template <typename T>
__device__ __forceinline__ void widen8(float *v, const typename Eight<T>::type &w)
{
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = (float)w[j];
}

template <typename T>
__device__ __forceinline__ void store8(T *row, const float *v, int col, int channels)
{
    typedef T V4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef T V2 __attribute__((ext_vector_type(2), aligned(sizeof(T))));
    typename Eight<T>::type w;
#pragma unroll
    for (int j = 0; j < 8; j++) w[j] = (T)v[j];
    if (col + 8 <= channels) {
        *(typename Eight<T>::type *)(row + col) = w;
        return;
    }
    const int n = channels - col;
    if (n <= 0) return;
    if (n & 4) *(V4 *)(row + col) = V4{w[0], w[1], w[2], w[3]};
    const V2 pair = (n & 4) ? V2{w[4], w[5]} : V2{w[0], w[1]}, next = (n & 4) ? V2{w[6], w[7]} : V2{w[2], w[3]};
    if (n & 2) *(V2 *)(row + col + (n & 4)) = pair;
    if (n & 1) row[col + (n & 6)] = (n & 2) ? next[0] : pair[0];
}

// exponents of a checkpoint as they are held, e + 127: the least of a type, and the one at which 64 2^e leaves its range
template <typename T> __device__ __forceinline__ constexpr uint32_t least_exponent() { return __is_same(T, f16) ? 103u : 1u; }
template <typename T> __device__ __forceinline__ constexpr uint32_t top_exponent() { return __is_same(T, f16) ? 137u : 249u; }

// Eight lanes hold a group of 64 channels, eight each: its exponent (0: not finite), and this lane's values as bytes.
template <typename T>
__device__ __forceinline__ uint32_t hold8(const float *v, uint2 &bytes)
{
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; j++) most = max(most, __float_as_uint(v[j]) & 0x7FFFFFFFu);          // (as whole numbers: NaN is above infinity)
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    // most = 2^E m with 1 <= m < 2: 2^(E - 6) if m < 127.5 / 64 (its upper mantissa bits are not all ones), else the next
    uint32_t e = (most >> 23) + ((most & 0x7F0000u) == 0x7F0000u ? 1u : 0u);
    e = max(e, least_exponent<T>() + 6u) - 6u;
    const bool finite = most < 0x7F800000u;
    const float by = __uint_as_float((254u - e) << 23), limit = e >= top_exponent<T>() ? 63.0f : 127.0f;
    bytes = make_uint2(0, 0);
    if (finite) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int q = (int)fminf(fmaxf(rintf(v[j] * by), -limit), limit);
            (j < 4 ? bytes.x : bytes.y) |= (uint32_t)(q & 255) << (8 * (j & 3));
        }
    }
    return finite ? e : 0u;
}

// the values of eight bytes under an exponent
__device__ __forceinline__ void held8(float *v, uint2 bytes, uint32_t e)
{
    const float by = e == 0u ? __uint_as_float(0x7FC00000u) : __uint_as_float(e << 23);
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = (float)(int8_t)((j < 4 ? bytes.x : bytes.y) >> (8 * (j & 3))) * by;
}

inline int launched(hipError_t e)
{
    if (e != hipSuccess) (void)hipGetLastError();
    return (int)e;
}

}  // namespace tessel
