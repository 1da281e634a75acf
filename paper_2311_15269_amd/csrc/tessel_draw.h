// Random words of a place and a number, and dropout by them (formulas: include/tessel_block_ops.h).  (Included by kernel sources only.)
#pragma once
#include "tessel_rows.h"

namespace tessel {

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011)
__device__ __forceinline__ uint4v philox(uint4v c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const uint64_t p = (uint64_t)c[0] * 0xD2511F53u, q = (uint64_t)c[2] * 0xCD9E8D57u;
        c = uint4v{(uint32_t)(q >> 32) ^ c[1] ^ k0, (uint32_t)q, (uint32_t)(p >> 32) ^ c[3] ^ k1, (uint32_t)p};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// the number that a kernel draws under
__device__ __forceinline__ uint64_t number_of(const DropLaunch &d) { return d.number + (d.step ? *d.step : 0); }

// dropout of the eight values from channel col (a multiple of 8) of a token on
__device__ __forceinline__ void drop8(float *v, const DropLaunch &d, uint64_t number, uint32_t token, int col)
{
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint4v w = philox(uint4v{(uint32_t)col / 4u + h, token, (uint32_t)number, (uint32_t)(number >> 32)}, (uint32_t)d.seed, (uint32_t)(d.seed >> 32));
#pragma unroll
        for (int j = 0; j < 4; j++) v[4 * h + j] = w[j] >= d.least ? v[4 * h + j] * d.by : 0.0f;
    }
}

#define BY_TYPE(type, call) ((type) == TESSEL_BF16 ? call(bf16) : (type) == TESSEL_F16 ? call(f16) : call(float))

}  // namespace tessel
