// What the kernels that hold a token row across threads share: sums over the
// row, and values formed again from stored words.
#pragma once

#include "q8.h"

namespace acsc {

// Sum over the wave, in every lane: rows of 16 by row_ror, then across rows.
__device__ __forceinline__ float wave_sum(float x)
{
#define ACSC_ROR(n) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + n, 0xF, 0xF, false))
    ACSC_ROR(8);
    ACSC_ROR(4);
    ACSC_ROR(2);
    ACSC_ROR(1);
#undef ACSC_ROR
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    return x;
}

// Sums over the NT threads of a row.  `slot` holds NT / 64 values per sum and
// is written once between two barriers of the caller's row loop.
template <int NT, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float *slot)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        s[i] = wave_sum(s[i]);
    if (NT > 64) {
        constexpr int W = NT / 64;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                slot[i * W + (threadIdx.x >> 6)] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w)
                s[i] += slot[i * W + w];
        }
    }
}

// Makes the compiler take what it knows of stored words as new: values are
// then formed from them again instead of being kept in registers.
template <int N>
__device__ __forceinline__ void again(uint32_t (&w)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        asm volatile("" : "+v"(w[i]));
}
template <int N>
__device__ __forceinline__ void again(float (&)[N])
{
}

}  // namespace acsc
