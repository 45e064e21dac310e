// Keyed draws for dropout: the chain over a mask key's fields and its mixers, by
// the rule that the iid boundary mask (ac.hip) follows too.
#pragma once

#include "common.h"

namespace acsc {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

// SplitMix64 output function (Steele, Lea & Flood 2014).
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// MurmurHash3 32-bit finaliser (Appleby).
__device__ __forceinline__ uint32_t fmix32(uint32_t h)
{
    h ^= h >> 16;
    h *= 0x85EBCA6Bu;
    h ^= h >> 13;
    h *= 0xC2B2AE35u;
    h ^= h >> 16;
    return h;
}

// Key chain over the fields of g(layer, step, B, S, H), plus seed and microbatch.
inline uint64_t chain_key(const ac_mask_key &k)
{
    uint64_t z = k.seed;
    for (const uint64_t f : {static_cast<uint64_t>(k.layer), k.step, static_cast<uint64_t>(k.microbatch),
                             static_cast<uint64_t>(k.B), static_cast<uint64_t>(k.S), static_cast<uint64_t>(k.H)})
        z = mix64((z ^ f) + kGamma);
    return z;
}

// Sixteen bits a value (rows' and columns' draws are iid): with k the row's
// key, a and b its low and high 32 bits, columns 2 q and 2 q + 1 take the low
// and the high 16 bits of this.
__device__ __forceinline__ uint32_t iid_pair(uint32_t a, uint32_t b, uint32_t q) { return fmix32(fmix32(a ^ q) ^ b); }

// T = floor(keep 65536 + 1/2): a value is kept where its 16 bits are below T.
inline int iid_threshold(double keep, uint32_t *T)
{
    ACSC_CHECK_ARG(keep > 0.0 && keep <= 1.0, ACSC_EINVAL, "keep=%g outside (0, 1]", keep);
    const double t = std::floor(keep * 65536.0 + 0.5);
    ACSC_CHECK_ARG(t >= 1.0, ACSC_EINVAL, "keep=%g rounds to a zero threshold (keep >= 2^-17)", keep);
    *T = static_cast<uint32_t>(t > 65536.0 ? 65536.0 : t);
    return ACSC_OK;
}

}  // namespace acsc
