// Random words of a place and a number, and dropout by them (formulas: include/tessel_block_ops.h).  (Included by kernel sources only.)
#pragma once
#include "tessel_rows.h"

namespace tessel {

// a product of 64 bits, by the one instruction for it (the compiler takes two, for each half; all of them run at the same rate)
__device__ __forceinline__ uint64_t wide_product(uint32_t a, uint32_t by)
{
    uint64_t r;
    asm("v_mad_u64_u32 %0, vcc, %1, %2, 0" : "=v"(r) : "v"(a), "s"(by) : "vcc");
    return r;
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// Dropout of eight neighbouring channels by Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
// A round takes words (a, b, c, d) to (hi(C c) ^ b ^ k, lo(C c), hi(A a) ^ d ^ m, lo(A a)).  Of the counter (column / 4, token, number) the token
// enters one word, so that a lane that keeps its columns works out once what the first three rounds make of them: five of six products.  A
// token that is the same for a whole wave is multiplied by the scalar unit.  Left for eight values: 30 products and 34 exclusive ors of two or three.
struct Draw {
    static constexpr uint32_t kA = 0xD2511F53u, kC = 0xCD9E8D57u, kK = 0x9E3779B9u, kM = 0xBB67AE85u;
    uint32_t least, k, m, first;                                 // (the same for all lanes)
    float    by;
    int      counters;           // one where a row has no more than four channels
    uint32_t b[2], c[2], d[2], e[2];                             // of the two counters, behind the second and third round
    __device__ __forceinline__ Draw(const DropLaunch &l, int channels, int col)
        : least(l.least), k((uint32_t)l.seed), m((uint32_t)(l.seed >> 32)), first(0), by(l.by), counters(channels > 4 ? 2 : 1)
    {
        if (least == 0) return;
        const uint64_t number = l.number + (l.step ? *l.step : 0), q = (uint64_t)(uint32_t)number * kC;
        first = (uint32_t)(q >> 32) ^ k;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint64_t p = wide_product((uint32_t)col / 4u + h, kA);
            const uint64_t r = wide_product((uint32_t)(p >> 32) ^ (uint32_t)(number >> 32) ^ m, kC);
            const uint64_t s = wide_product((uint32_t)(r >> 32) ^ (uint32_t)q ^ (k + kK), kA);
            b[h] = (uint32_t)p ^ (m + kM);
            c[h] = (uint32_t)r ^ (k + 2 * kK);
            d[h] = (uint32_t)(s >> 32) ^ (m + 2 * kM);
            e[h] = (uint32_t)s;
        }
    }
    // eight values of a token, behind a look at `least`
    __device__ __forceinline__ void apply(float *v, uint32_t token) const
    {
        const uint64_t p = (uint64_t)(first ^ token) * kA;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            if (h >= counters) break;
            const uint64_t q = wide_product((uint32_t)(p >> 32) ^ b[h], kC);
            uint32_t w[4] = {(uint32_t)(q >> 32) ^ c[h], (uint32_t)q, d[h] ^ (uint32_t)p, e[h]};
#pragma unroll
            for (int i = 3; i < 10; i++) {
                const uint64_t x = wide_product(w[0], kA), y = wide_product(w[2], kC);
                w[0] = xor3((uint32_t)(y >> 32), w[1], k + i * kK);
                w[2] = xor3((uint32_t)(x >> 32), w[3], m + i * kM);
                w[1] = (uint32_t)y;
                w[3] = (uint32_t)x;
            }
#pragma unroll
            for (int j = 0; j < 4; j++) v[4 * h + j] = w[j] >= least ? v[4 * h + j] * by : 0.0f;
        }
    }
};

// Eight values of a row without a branch around the read, and put in their places behind all reads (tessel_rows.h); rows of fewer than eight, which a
// NARROW kernel may have, in pieces of four, two and one.
template <typename T, bool NARROW>
__device__ __forceinline__ typename Eight<T>::type read8(const T *row, int col, int channels)
{
    if (NARROW && channels < 8) return raw8<T>(row, col, channels);
    return take8<T, false>(row, col, channels);
}
template <typename T, bool NARROW>
__device__ __forceinline__ void place8(int col, int channels, typename Eight<T>::type &x)
{
    if (!NARROW || channels >= 8) settle8<T, false>(col, channels, x);
}

// The places of a wave in [tokens][channels], ROWS tokens a lane: WIDE, 64 chunks of eight channels of the same tokens (a wave for each tile of 512 channels);
// else 64 / lanes tokens at a time, `lanes` a power of two.
template <bool WIDE, int ROWS>
struct Span {
    int     col;
    int64_t token;               // the first of the lane's
    int     step;                // from one to the next
    __device__ __forceinline__ Span(int channels, int lanes)
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (blockDim.x / 64) + threadIdx.x / 64), lane = threadIdx.x & 63;
        if constexpr (WIDE) {
            const uint32_t tiles = ((uint32_t)channels + 511u) / 512u, group = wave / tiles;
            col = (int)(wave - group * tiles) * 512 + 8 * lane;
            token = (int64_t)group * ROWS;
            step = 1;
        } else {
            step = 64 / lanes;
            col = 8 * (lane % lanes);
            token = (int64_t)wave * step * ROWS + lane / lanes;
        }
    }
};
// chunks of eight channels that a row takes up to 64 lanes for, and the workgroups of 256 of such a launch
struct SpanShape {
    bool    wide;
    int     lanes;
    int64_t groups;
};
inline SpanShape span_shape(int64_t tokens, int channels, int rows)
{
    SpanShape s = {channels > 256, 1, 0};
    while (s.lanes < 64 && 8 * s.lanes < channels) s.lanes *= 2;
    const int64_t at_once = (int64_t)(64 / s.lanes) * rows, tiles = s.wide ? ((int64_t)channels + 511) / 512 : 1;
    s.groups = ((tokens + at_once - 1) / at_once * tiles + 3) / 4;
    return s;
}
// Tokens a lane: four where dropout of 16-bit values would else hold memory up, as their columns are worked out once for all, or where a launch does not hold the threads for one
// (a row's lanes are up to twice its chunks, of which there are at most 2^32); else one.  The lookup's reads wait for its tokens, a dropout's for nothing, which so gains in rows of up
// to 256 channels alone (`widest`).  By fours and by ones, every call on other memory, 2^22 chunks of bf16: dropout of rows of 1 channel 17.2 and 20.9 us, 9: 27.8 and 30.4, 256: 27.3
// and 28.0, 4096: 27.7 and 26.6 (a pass of two, waited for: 62.7 and 63.4); lookup with dropout of rows of 64 27.6 and 32.3, 4096: 28.7 and 30.4.  2^24 x 1: 57 and 74.  Of 2^20 chunks fours are the
// same or up to 14 % slower, of 2^21 15 % faster to 13 % slower by width and operator, in 32 bits some 5 % slower.
inline int span_rows(int type, int64_t tokens, int channels, const DropLaunch &d, int widest)
{
    const bool held_up = d.least && type != TESSEL_F32 && channels <= widest && tokens * (((int64_t)channels + 7) / 8) >= 1 << 22;
    return held_up || span_shape(tokens, channels, 1).groups > UINT32_MAX / 256 ? 4 : 1;
}

#define BY_TYPE(type, call) ((type) == TESSEL_BF16 ? call(bf16) : (type) == TESSEL_F16 ? call(f16) : call(float))

}  // namespace tessel
